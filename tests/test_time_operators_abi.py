"""What the operators along time refuse, on the host before anything is launched (no call here needs a GPU)."""
import ctypes
import itertools
import os
import random

import pytest
import torch

from paper_2504_11681_amd import binding as tfno

FAKE = 0x10000000      # never dereferenced: every call fails its checks, or has nothing to do
MB = 1 << 20


@pytest.fixture(scope="module")
def L():
    from paper_2504_11681_amd import build
    if not os.path.exists(tfno.LIB_PATH) or not os.path.exists(build.MARSHAL):
        build.build(verbose=False)
    return tfno.lib()


def strides(T, H, D):
    return tfno._Strides(T * H * D, H * D, D)


def norm_desc(**kw):
    d = tfno._HeadNormDesc(1, 2, 8, 4, 2, 64, 32, 8, 0, 1e-6, 0)
    for n, H in (("q", 4), ("k", 2), ("q_out", 4), ("k_out", 2), ("dq", 4), ("dk", 2)):
        setattr(d, n, strides(8, H, 64))
    for n, v in kw.items():
        setattr(d, n, v)
    return d


def rule_desc(**kw):
    d = tfno._DeltaRuleDesc(1, 2, 8, 2, 4, 64, 64, 0.125)
    for n, H, D in (("q", 2, 64), ("k", 2, 64), ("v", 4, 64), ("o", 4, 64), ("g", 4, 1), ("beta", 4, 1), ("dq", 2, 64), ("dk", 2, 64), ("dv", 4, 64),
                    ("dg", 4, 1), ("dbeta", 4, 1)):
        setattr(d, n, strides(8, H, D))
    for n, v in kw.items():
        setattr(d, n, v)
    return d


def call(fn, desc, args, **kw):
    a = dict(args, **kw)
    return fn(ctypes.addressof(desc) if desc is not None else None, *a.values(), None)


def pointers(*names):
    return {n: FAKE + i * MB for i, n in enumerate(names)}


NORM = pointers("q", "k", "wq", "wk", "cos", "sin", "positions", "q_out", "k_out")
NORM_BACK = pointers("q", "k", "wq", "wk", "cos", "sin", "positions", "dq_out", "dk_out", "dq", "dk", "dwq", "dwk")
RULE = pointers("q", "k", "v", "g", "beta", "lengths", "initial", "o", "final", "tape")
RULE_BACK = pointers("q", "k", "v", "g", "beta", "lengths", "initial", "tape", "d_o", "d_final", "dq", "dk", "dv", "dg", "dbeta", "d_initial")


def test_norm_refuses(L):
    for fn, args, needed in ((L.tfno_head_norm_rope, NORM, ("q", "k", "cos", "sin", "q_out", "k_out")),
                             (L.tfno_head_norm_rope_backward, NORM_BACK, ("q", "k", "cos", "sin", "dq_out", "dk_out", "dq", "dk"))):
        assert call(fn, None, args) == tfno.ERR_NULL
        for n in needed:
            assert call(fn, norm_desc(), args, **{n: None}) == tfno.ERR_NULL, n
        for bad in (dict(dtype=2), dict(dtype=-1), dict(B=-1), dict(T=-1), dict(Hq=-1), dict(Hq=0, Hk=0), dict(D=0), dict(D=513), dict(R=-2), dict(R=3),
                    dict(R=66), dict(eps=0.0), dict(eps=float("nan")), dict(P=-1), dict(positions_batch=-1), dict(B=1 << 30, T=1 << 10),
                    dict(q=tfno._Strides(-1, 256, 64)), dict(k=tfno._Strides(1 << 40, 128, 64))):
            assert call(fn, norm_desc(**bad), args) == tfno.ERR_SHAPE, bad
        assert call(fn, norm_desc(P=7), args, positions=None) == tfno.ERR_SHAPE
        for n in needed:
            assert call(fn, norm_desc(), args, **{n: args[n] + 1}) == tfno.ERR_ALIGN, n
        assert call(fn, norm_desc(), args, cos=args["cos"] + 2) == tfno.ERR_ALIGN
        assert call(fn, norm_desc(B=0), dict.fromkeys(args)) == tfno.OK
        first, second = ("q_out", "k_out") if fn is L.tfno_head_norm_rope else ("dq", "dk")
        assert call(fn, norm_desc(), args, **{first: args[second]}) == tfno.ERR_ALIAS          # results over each other
        assert call(fn, norm_desc(), args, **{first: args["cos"]}) == tfno.ERR_ALIAS
        assert call(fn, norm_desc(), args, **{first: args["q"] + 2}) == tfno.ERR_ALIAS         # in place, but not at the same place
        assert call(fn, norm_desc(**{first: tfno._Strides(8 * 256, 256, 32)}), args) == tfno.ERR_ALIAS   # heads that overlap each other
        assert call(fn, norm_desc(**{first: tfno._Strides(0, 256, 64)}), args) == tfno.ERR_ALIAS         # one place for the whole batch


def test_norm_gradient_needs_its_workspace(L):
    need = L.tfno_head_norm_rope_workspace_bytes(64)
    assert need > 0 and L.tfno_head_norm_rope_workspace_bytes(0) == 0 and L.tfno_head_norm_rope_workspace_bytes(513) == 0
    assert L.tfno_set_workspace(None, 0) == tfno.OK
    assert call(L.tfno_head_norm_rope_backward, norm_desc(), NORM_BACK) == tfno.ERR_WORKSPACE
    assert L.tfno_set_workspace(FAKE + 64 * MB, need - 1) == tfno.OK
    assert call(L.tfno_head_norm_rope_backward, norm_desc(), NORM_BACK) == tfno.ERR_WORKSPACE
    assert L.tfno_set_workspace(NORM_BACK["dq_out"], need) == tfno.OK
    assert call(L.tfno_head_norm_rope_backward, norm_desc(), NORM_BACK) == tfno.ERR_ALIAS
    assert L.tfno_set_workspace(None, 0) == tfno.OK


def test_rule_refuses(L):
    for fn, args, needed, outputs in (
            (L.tfno_gated_delta_rule, RULE, ("q", "k", "v", "beta", "o"), ("o", "final", "tape")),
            (L.tfno_gated_delta_rule_backward, RULE_BACK, ("q", "k", "v", "beta", "tape", "d_o", "dq", "dk", "dv", "dbeta"), ("dq", "dk", "dv", "dg", "dbeta", "d_initial"))):
        assert call(fn, None, args) == tfno.ERR_NULL
        for n in needed:
            assert call(fn, rule_desc(), args, **{n: None}) == tfno.ERR_NULL, n
        for bad in (dict(dtype=2), dict(B=-1), dict(T=-1), dict(Hk=0), dict(Hv=0), dict(Hv=3), dict(Dk=0), dict(Dv=0), dict(q=tfno._Strides(1024, -128, 64)),
                    dict(v=tfno._Strides(1 << 41, 256, 64)), dict(B=1 << 20, Hk=64, Hv=64), dict(T=2147483647, B=4)):
            assert call(fn, rule_desc(**bad), args) == tfno.ERR_SHAPE, bad
        for bad in (dict(Dk=129), dict(Dv=257)):
            assert call(fn, rule_desc(**bad), args) == tfno.ERR_UNSUPPORTED, bad
        for n in args:
            if n != "tape":
                assert call(fn, rule_desc(), args, **{n: args[n] + 1}) == tfno.ERR_ALIGN, n
        assert call(fn, rule_desc(), args, tape=args["tape"] + 128) == tfno.ERR_ALIGN
        for n in outputs:
            other = "k" if n != "tape" else "q"
            assert call(fn, rule_desc(), args, **{n: args[other]}) == tfno.ERR_ALIAS, n
        assert call(fn, rule_desc(**{"o" if fn is L.tfno_gated_delta_rule else "dv": tfno._Strides(2048, 0, 64)}), args) == tfno.ERR_ALIAS
        assert call(fn, rule_desc(B=0), dict.fromkeys(args)) == tfno.OK
        assert call(fn, rule_desc(T=0), dict.fromkeys(args)) == tfno.OK


def test_slices_of_one_projection_are_no_aliases(L):
    """q, k, v and the result interleaved in rows of one buffer: refused for the workspace alone; one value closer together, as an alias."""
    d = rule_desc()
    for n, H in (("q", 2), ("k", 2), ("v", 4), ("o", 4)):
        setattr(d, n, tfno._Strides(8 * 12 * 64, 12 * 64, 64))
    at = dict(RULE, q=FAKE, k=FAKE + 2 * 128, v=FAKE + 4 * 128, o=FAKE + 8 * 128, tape=None)
    assert L.tfno_set_workspace(None, 0) == tfno.OK
    assert call(L.tfno_gated_delta_rule, d, at) == tfno.ERR_WORKSPACE
    assert call(L.tfno_gated_delta_rule, d, at, o=FAKE + 8 * 128 - 2) == tfno.ERR_ALIAS
    assert call(L.tfno_gated_delta_rule, d, at, o=FAKE + 8 * 128 + 2) == tfno.ERR_ALIAS


    # one buffer [B, 4, T, H, D]
    for n, H in (("q", 2), ("k", 2), ("v", 4), ("o", 4)):
        setattr(d, n, tfno._Strides(4 * 8 * 256, H * 64, 64))
    at = dict(RULE, q=FAKE, k=FAKE + 2 * 8 * 256, v=FAKE + 4 * 8 * 256, o=FAKE + 6 * 8 * 256, tape=None)
    assert call(L.tfno_gated_delta_rule, d, at) == tfno.ERR_WORKSPACE
    assert call(L.tfno_gated_delta_rule, d, at, o=FAKE + 6 * 8 * 256 - 2) == tfno.ERR_ALIAS
    assert call(L.tfno_gated_delta_rule, d, at, o=FAKE + 6 * 8 * 256 + 2) == tfno.ERR_ALIAS


def elements(at, elem, sizes, strides, D):
    """Addresses of all bytes of a tensor."""
    first = [at + elem * sum(i * s for i, s in zip(index, strides)) for index in itertools.product(*map(range, sizes))]
    return {x + y for x in first for y in range(elem * D)}


def pair_layout(order, sizes, D):
    """Strides (batch, token, head) and the distance of two tensors of one buffer whose axes, from the outermost on, are `order`, D values last."""
    step, at = D, {}
    for axis in reversed(order):
        at[axis] = step
        step *= sizes[axis]
    return tfno._Strides(at["batch"], at["token"], at["head"]), at["slot"]


@pytest.mark.parametrize("sizes", [dict(batch=2, token=8, head=4, slot=2), dict(batch=1, token=8, head=4, slot=3), dict(batch=3, token=1, head=4, slot=2),
                                   dict(batch=2, token=5, head=1, slot=2), dict(batch=1, token=1, head=4, slot=2)])
@pytest.mark.parametrize("order", list(itertools.permutations(("batch", "token", "head", "slot"))))
def test_slices_that_interleave_along_any_axis_are_no_aliases(L, order, sizes):
    """v and o, d_o and dv, dg and dbeta, dq and dk in place of q and k: slices of one buffer in every order of the axes.  They are refused for the workspace alone, and as aliases
    when one lies an element closer to the other."""
    assert L.tfno_set_workspace(None, 0) == tfno.OK
    B, T, H = sizes["batch"], sizes["token"], sizes["head"]
    s, far = pair_layout(order, sizes, 64)
    shape = dict(B=B, T=T, Hk=H, Hv=H, **{n: strides(T, H, 64) for n in ("q", "k", "dq", "dk")}, **{n: strides(T, H, 1) for n in ("g", "beta")})
    d = rule_desc(**shape, v=s, o=s)
    at = dict(RULE, v=FAKE + 200 * MB, o=FAKE + 200 * MB + 2 * far, tape=None)
    assert call(L.tfno_gated_delta_rule, d, at) == tfno.ERR_WORKSPACE
    assert call(L.tfno_gated_delta_rule, d, at, o=at["o"] - 2) == tfno.ERR_ALIAS
    gates, near = pair_layout(order, sizes, 1)
    d = rule_desc(**shape, dg=gates, dbeta=gates, dv=s, o=s)
    at = dict(RULE_BACK, tape=FAKE + 400 * MB, d_o=FAKE + 200 * MB, dv=FAKE + 200 * MB + 2 * far, dg=FAKE + 300 * MB, dbeta=FAKE + 300 * MB + 4 * near)
    assert call(L.tfno_gated_delta_rule_backward, d, at) == tfno.ERR_WORKSPACE
    assert call(L.tfno_gated_delta_rule_backward, d, at, dv=at["dv"] - 2) == tfno.ERR_ALIAS
    assert call(L.tfno_gated_delta_rule_backward, d, at, dbeta=at["dbeta"] - 4) == tfno.ERR_ALIAS
    n = norm_desc(B=B, T=T, Hq=H, Hk=H, P=T, q=s, k=s, dq=s, dk=s, q_out=strides(T, H, 64), k_out=strides(T, H, 64))
    at = dict(NORM_BACK, q=FAKE + 200 * MB, k=FAKE + 200 * MB + 2 * far, positions=None)
    at["dq"], at["dk"] = at["q"], at["k"]
    assert call(L.tfno_head_norm_rope_backward, n, at) == tfno.ERR_WORKSPACE
    assert call(L.tfno_head_norm_rope_backward, n, at, dk=at["k"] - 2) == tfno.ERR_ALIAS


def test_strides_of_axes_of_one_do_not_count_in_place(L):
    assert L.tfno_set_workspace(None, 0) == tfno.OK
    n = norm_desc(T=1, q=tfno._Strides(256, 1 << 20, 64), dq=tfno._Strides(256, 256, 64))
    assert call(L.tfno_head_norm_rope_backward, n, dict(NORM_BACK, dq=NORM_BACK["q"])) == tfno.ERR_WORKSPACE


def test_tensors_that_share_bytes_are_always_aliases(L):
    """Small tensors of random strides at random places close to each other, against the sets of their bytes."""
    assert L.tfno_set_workspace(None, 0) == tfno.OK
    rng, shared, free = random.Random(5), 0, 0
    for _ in range(4000):
        B, T, H, D = rng.randint(1, 3), rng.randint(1, 4), rng.randint(1, 3), rng.choice((1, 2, 3, 8))
        unit = rng.choice((1, D, 2 * D, 3 * D))

        def random_strides():
            return tuple(unit * rng.choice((0, 1, 2, 3, 4, 6, 8, 12, 24)) for _ in range(3))

        sv, so, off = random_strides(), random_strides(), 2 * rng.randint(0, 40)
        d = rule_desc(B=B, T=T, Hk=1, Hv=H, Dv=D, v=tfno._Strides(*sv), o=tfno._Strides(*so), q=strides(T, 1, 64), k=strides(T, 1, 64), g=strides(T, H, 1), beta=strides(T, H, 1))
        at = dict(RULE, v=FAKE + 200 * MB, o=FAKE + 200 * MB + off, tape=None)
        st = call(L.tfno_gated_delta_rule, d, at)
        v, o = elements(at["v"], 2, (B, T, H), sv, D), elements(at["o"], 2, (B, T, H), so, D)
        if v & o or len(o) < 2 * B * T * H * D:
            assert st == tfno.ERR_ALIAS, (B, T, H, D, sv, so, off)
            shared += 1
        else:
            free += st == tfno.ERR_WORKSPACE
    assert shared > 500 and free > 200, (shared, free)


def test_rule_memory(L):
    d = rule_desc()
    tape, forward, backward = L.tfno_gated_delta_rule_tape_bytes(ctypes.addressof(d)), *(L.tfno_gated_delta_rule_workspace_bytes(ctypes.addressof(d), b) for b in (0, 1))
    assert tape > forward > 0 and backward > 0
    longer = rule_desc(T=8 * 64)
    assert L.tfno_gated_delta_rule_tape_bytes(ctypes.addressof(longer)) >= 7 * tape
    for bad in (dict(Dk=129), dict(Hv=3), dict(B=-1)):
        bad = rule_desc(**bad)
        assert L.tfno_gated_delta_rule_tape_bytes(ctypes.addressof(bad)) == 0
        assert L.tfno_gated_delta_rule_workspace_bytes(ctypes.addressof(bad), 1) == 0
    assert L.tfno_set_workspace(None, 0) == tfno.OK
    assert call(L.tfno_gated_delta_rule, d, RULE, tape=None) == tfno.ERR_WORKSPACE
    assert call(L.tfno_gated_delta_rule_backward, d, RULE_BACK) == tfno.ERR_WORKSPACE
    assert L.tfno_set_workspace(FAKE + 64 * MB, forward - 1) == tfno.OK
    assert call(L.tfno_gated_delta_rule, d, RULE, tape=None) == tfno.ERR_WORKSPACE
    assert L.tfno_set_workspace(RULE["q"], forward) == tfno.OK
    assert call(L.tfno_gated_delta_rule, d, RULE, tape=None) == tfno.ERR_ALIAS
    assert L.tfno_set_workspace(None, 0) == tfno.OK


def test_step_refuses(L):
    args = pointers("q", "k", "v", "g", "beta", "states", "slots", "pool", "o")
    args["pool"] = 5
    args["states"] = FAKE + 100 * MB
    fn, d = L.tfno_gated_delta_rule_step, lambda **kw: rule_desc(**{"T": 1, **kw})
    assert call(fn, None, args) == tfno.ERR_NULL
    for n in ("q", "k", "v", "beta", "states", "o"):
        assert call(fn, d(), args, **{n: None}) == tfno.ERR_NULL, n
    for bad in (dict(T=2), dict(T=0), dict(Hv=5), dict(dtype=7), dict(B=-2)):
        assert call(fn, d(**bad), args) == tfno.ERR_SHAPE, bad
    assert call(fn, d(), args, pool=-1) == tfno.ERR_SHAPE
    assert call(fn, d(), args, slots=None, pool=1) == tfno.ERR_SHAPE
    assert call(fn, d(Dk=200), args) == tfno.ERR_UNSUPPORTED
    for n in ("q", "k", "v", "g", "beta", "states", "slots", "o"):
        assert call(fn, d(), args, **{n: args[n] + 1}) == tfno.ERR_ALIGN, n
    assert call(fn, d(), args, o=args["states"]) == tfno.ERR_ALIAS
    assert call(fn, d(), args, v=args["states"]) == tfno.ERR_ALIAS
    assert call(fn, d(B=0), args) == tfno.OK


def test_binding_refuses_what_is_not_on_the_device_or_has_another_type():
    q = torch.zeros(2, 8, 2, 16)          # on the CPU
    g = torch.zeros(2, 8, 2)
    with pytest.raises(TypeError):
        tfno.gated_delta_rule(q, q, q, g, g, q)
    with pytest.raises(TypeError):
        tfno.gated_delta_rule(q, q.double(), q, g, g, q)
    with pytest.raises(TypeError):
        tfno.gated_delta_rule(q, q, q, g.double(), g, q)
    with pytest.raises(TypeError):
        tfno.head_norm_rope(q, q.bfloat16(), None, None, None, None, q, q)
    with pytest.raises(TypeError):
        tfno.head_norm_rope(q, q, None, None, None, None, q, q, positions=torch.zeros(2, 8))
    with pytest.raises(TypeError):
        tfno.gated_delta_rule_step(q[:, 0], q[:, 0], q[:, 0], g[:, 0], g[:, 0], torch.zeros(2, 2, 16, 16), q[:, 0], slots=torch.zeros(2))


def plans(*tensors):
    """What a plan depends on of these tensors, as if they lay on device 0."""
    return [None if t is None else (t.dtype, 0, t.shape, t.stride()) for t in tensors]


def test_binding_refuses_shapes_that_do_not_fit():
    q, v, g = torch.zeros(2, 8, 2, 16), torch.zeros(2, 8, 4, 24), torch.zeros(2, 8, 4)
    none = [None] * 10
    good = (q, q, v, v, g, g)
    plan = tfno._rule_plan(*plans(*good), *none, None)
    assert plan[-1].scale == 0.25 and plan[1] > plan[2] > 0
    for bad in ((q[:, :7], q, v, v, g, g), (q, q[..., :8], v, v, g, g), (q, q, v, q, g, g), (q, q, v, v, g[..., :2], g), (q, q, v, v, g, g[:1]), (q[0], q[0], v, v, g, g),
                (q, q, v, v.transpose(2, 3), g, g)):
        with pytest.raises(ValueError):
            tfno._rule_plan(*plans(*bad), *none, None)
    with pytest.raises(ValueError):      # the last axis has to be contiguous
        tfno._rule_plan(*plans(torch.zeros(2, 8, 2, 32)[..., ::2], q, v, v, g, g), *none, None)
    with pytest.raises(TypeError):
        tfno._rule_plan(*plans(q.half(), q.half(), v.half(), v.half(), g, g), *none, None)
    with pytest.raises(TypeError):
        tfno._rule_plan(*plans(q, q.double(), v, v, g, g), *none, None)
    with pytest.raises(TypeError):
        tfno._rule_plan(*plans(q, q, v, v, g, g.double()), *none, None)
    more = dict(lengths=torch.zeros(2, dtype=torch.int32), tape=torch.zeros(plan[1], dtype=torch.uint8), initial=torch.zeros(2, 4, 16, 24), final=torch.zeros(2, 4, 16, 24),
                other=torch.zeros(2, 4, 16, 24))

    def with_more(**kw):
        return tfno._rule_plan(*plans(*good), *[None] * 5, *plans(*{**more, **kw}.values()), None)

    assert with_more()[1] == plan[1]
    for kw in (dict(lengths=torch.zeros(3, dtype=torch.int32)), dict(tape=more["tape"][1:]), dict(tape=torch.zeros(2, plan[1], dtype=torch.uint8)),
               dict(initial=torch.zeros(2, 4, 24, 16)), dict(final=torch.zeros(2, 4, 24, 16).transpose(2, 3)), dict(other=torch.zeros(1, 4, 16, 24))):
        with pytest.raises(ValueError):
            with_more(**kw)
    for kw in (dict(lengths=torch.zeros(2)), dict(tape=torch.zeros(plan[1])), dict(initial=torch.zeros(2, 4, 16, 24, dtype=torch.bfloat16))):
        with pytest.raises(TypeError):
            with_more(**kw)


def test_binding_refuses_shapes_of_the_norm_and_the_step_that_do_not_fit():
    q, v, g = torch.zeros(2, 8, 2, 16), torch.zeros(2, 8, 4, 24), torch.zeros(2, 8, 4)
    w, cos = torch.zeros(16), torch.zeros(8, 4)

    def norm(q, k, w, cos, sin, positions=None):
        return tfno._head_norm_plan(*plans(q, k, q, k, None, None, positions, w, w, None, None, cos, sin), 1e-6, False)

    assert norm(q, q, w, cos, cos)[-1].R == 8
    for bad in ((q, q[:1], w, cos, cos), (q, q[..., :8], w, cos, cos), (q, q, w[:8], cos, cos), (q, q, w, cos[0], cos[0]), (q[0], q[0], w, cos, cos), (q, q, w, cos, None),
                (q, q, torch.zeros(32)[::2], cos, cos), (q, q, w, cos, cos[:4]), (q, q, w, cos, cos, torch.zeros(2, 7, dtype=torch.int32)),
                (q, q, w, torch.zeros(8, 8)[:, ::2], cos)):
        with pytest.raises(ValueError):
            norm(*bad)
    with pytest.raises(TypeError):
        norm(q, q, w, cos, cos, torch.zeros(2, 8))
    s, slots = torch.zeros(3, 4, 16, 24), torch.zeros(2, dtype=torch.int32)

    def step(states, slots=None, o=v[:, 0], beta=g[:, 0]):
        return tfno._step_plan(*plans(q[:, 0], q[:, 0], v[:, 0], o, g[:, 0], beta, states, slots), None)

    assert step(s, slots)[-1].T == 1
    for bad in ((s[:, :2],), (s[0],), (s[..., :8],), (s, torch.zeros(3, dtype=torch.int32)), (s, slots, v[:1, 0]), (s, slots, v[:, 0], g[:, 0, :2]), (s.transpose(2, 3).contiguous(),)):
        with pytest.raises(ValueError):
            step(*bad)
    with pytest.raises(TypeError):
        step(s, torch.zeros(2))


def test_rule_says_which_distances_it_does_not_support(L):
    """Tokens of v, o and their gradients are walked with 32-bit offsets inside a chunk: their distance is below 2^24 elements."""
    far = tfno._Strides(1 << 30, 1 << 24, 64)
    for n in ("v", "o"):
        assert call(L.tfno_gated_delta_rule, rule_desc(**{n: far}), RULE) == tfno.ERR_UNSUPPORTED, n
    for n in ("o", "dv"):            # the gradient is taken from the tape, which holds what it needs of v
        assert call(L.tfno_gated_delta_rule_backward, rule_desc(**{n: far}), RULE_BACK) == tfno.ERR_UNSUPPORTED, n


def test_sizes_that_no_launch_takes_are_refused(L):
    """A launch takes less than 2^32 threads.  A walk of 256 columns has 1280 a head: 2^21 heads of a sequence are taken, 2^23 are not; of a batch, pieces are."""
    assert L.tfno_set_workspace(None, 0) == tfno.OK
    for n, T, status in ((1 << 21, 1, tfno.ERR_WORKSPACE), (1 << 23, 1, tfno.ERR_SHAPE), (1 << 23, 0, tfno.ERR_SHAPE), (1 << 25, 0, tfno.ERR_SHAPE)):
        far = {m: FAKE + (i << 36) for i, m in enumerate(("q", "k", "v", "g", "beta", "lengths", "initial", "o", "final", "tape"))}
        d = rule_desc(B=1, T=T, Hk=1, Hv=n, Dk=1, Dv=256, v=strides(T, n, 256), o=strides(T, n, 256), g=strides(T, n, 1), beta=strides(T, n, 1))
        assert call(L.tfno_gated_delta_rule, d, far, tape=None) == status, (n, T)
        if status != tfno.ERR_SHAPE:
            d.B, d.Hk, d.Hv = 16 * n, 1, 1
            for m in ("v", "o"):
                setattr(d, m, strides(T, 1, 256))
            for m in ("q", "k", "g", "beta"):
                setattr(d, m, strides(T, 1, 1))
            assert call(L.tfno_gated_delta_rule, d, far, tape=None) == status


def test_the_library_is_built_without_torch_and_whatever_becomes_of_the_calls_from_python(monkeypatch, capsys):
    import sys
    from paper_2504_11681_amd import build
    ran = []

    def run(cmd, what):
        ran.append(what)
        if what == "marshal.cpp":
            raise RuntimeError("no headers")

    monkeypatch.setattr(build, "_compile", lambda src: src + ".o")
    monkeypatch.setattr(build, "_run", run)
    with pytest.raises(RuntimeError, match="no headers"):
        build.build()
    assert sorted(ran) == ["link", "marshal.cpp"]
    ran.clear()
    monkeypatch.setitem(sys.modules, "torch", None)
    assert build.build() == build.LIB and ran == ["link"]
    assert "no _marshal.so" in capsys.readouterr().err


def test_key_holds_all_that_a_plan_depends_on(L):
    m = tfno._load_marshal()
    x = torch.zeros(2, 3, 4)
    keys = [m.key(t) for t in (x, x.bfloat16(), x.int(), x.byte(), x[:1], x[:, :0], x.transpose(0, 1), x.expand(2, 3, 4).as_strided((2, 3, 4), (0, 4, 1)),
                               x.as_strided((1, 3, 4), (1 << 40, 4, 1)), x[0], x[0, 0], x[0, 0, 0], None)]
    keys += [m.key(), m.key(x, None), m.key(None, x), m.key(x, x), m.key(None, None)]
    assert len(set(keys)) == len(keys)
    assert m.key(x, None) == m.key(torch.ones(2, 3, 4), None)


def test_what_is_no_tensor_or_has_no_memory_of_its_own_values_is_refused(L):
    m = tfno._load_marshal()
    x = torch.zeros(2, 8, 2, 64, dtype=torch.complex64)
    for bad, error in ((1.0, TypeError), ("x", TypeError), (x.conj(), ValueError), (x.conj().imag, ValueError), (x.real.to_sparse(), ValueError),
                       (torch.zeros((1,) * 9), ValueError)):
        with pytest.raises(error):
            m.key(bad)
    with pytest.raises(TypeError):
        m.tfno_gated_delta_rule_step(None)
    q = torch.zeros(2, 8, 2, 64)
    with pytest.raises(TypeError):                       # not on a GPU
        tfno.head_norm_rope(q, q, None, None, None, None, q, q)
    with pytest.raises((TypeError, AttributeError)):
        tfno.gated_delta_rule(None, None, None, None, None, None)


def test_workspace_of_large_batches_is_that_of_a_piece(L):
    """Without a tape a large batch goes through in pieces that share one workspace; its size does not grow with the batch, nor does a call ask for less than a piece."""
    def need(**kw):
        d = rule_desc(Hk=2, Hv=2, T=1024, **kw)
        return L.tfno_gated_delta_rule_workspace_bytes(ctypes.addressof(d), 0)

    sizes = [need(B=B) for B in (1, 64, 128, 256, 1024, 4096)]
    assert all(x > 0 for x in sizes) and sizes[1] < sizes[2] and sizes[3] < 2 * sizes[2] and sizes[5] == sizes[4] == sizes[3]
    assert need(B=150) > sizes[2] and need(B=257) >= sizes[2]
    assert need(B=1, Dk=128) > 0 and need(B=0) == 0
