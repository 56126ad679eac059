"""What the operators of a block along time refuse, on the host before anything is launched (no call here needs a GPU)."""
import ctypes
import math
import os

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


@pytest.fixture
def workspace(L):
    """One that is large enough for every call here, and behind all that they name."""
    assert L.tfno_set_workspace(FAKE + (1 << 32), 1 << 30) == tfno.OK
    yield
    assert L.tfno_set_workspace(None, 0) == tfno.OK


def pointers(*names):
    return {n: FAKE + i * MB for i, n in enumerate(names)}


def call(fn, desc, args, **kw):
    a = dict(args, **kw)
    return fn(ctypes.addressof(desc) if desc is not None else None, *a.values(), None)


def recurrence_desc(**kw):
    d = tfno._RecurrenceDesc(1, 2, 8, 64, 1)
    for n in ("x", "gate", "input_gate", "y", "dx", "dgate", "dinput_gate"):
        setattr(d, n, tfno._Strides(8 * 64, 64, 0))
    for n, v in kw.items():
        setattr(d, n, v)
    return d


def norm_desc(**kw):
    d = tfno._BlockNormDesc(1, 0, 2, 8, 64, 1, 1, 1, 1.0, 1e-6)
    for n in ("y", "r", "gate", "r_out", "n_out", "dy", "dr", "dgate"):
        setattr(d, n, tfno._Strides(8 * 64, 64, 0))
    for n, v in kw.items():
        setattr(d, n, v)
    return d


FORWARD = pointers("x", "gate", "input_gate", "rate", "lengths", "initial", "y", "final", "tape")
BACKWARD = pointers("x", "gate", "input_gate", "rate", "lengths", "tape", "d_y", "d_final", "dx", "dgate", "dinput_gate", "drate", "d_initial")
NORM = pointers("y", "r", "gate", "w_after", "w_before", "lengths", "r_out", "n_out")
NORM_BACK = pointers("y", "r", "gate", "w_after", "w_before", "lengths", "d_r_out", "d_n_out", "dy", "dr", "dgate", "dw_after", "dw_before")


def test_recurrence_refuses(L, workspace):
    for fn, args, needed in ((L.tfno_gated_recurrence, FORWARD, ("x", "gate", "y")),
                             (L.tfno_gated_recurrence_backward, BACKWARD, ("x", "gate", "tape", "d_y", "dx", "dgate", "dinput_gate"))):
        assert call(fn, None, args) == tfno.ERR_NULL
        for n in needed:
            assert call(fn, recurrence_desc(), args, **{n: None}) == tfno.ERR_NULL, n
        for bad in (dict(dtype=2), dict(dtype=-1), dict(B=-1), dict(T=-1), dict(C=0), dict(T=(1 << 30) + 1), dict(C=(1 << 28) + 1), dict(B=1 << 20, C=1 << 20), dict(B=(1 << 31) - 1, C=33),
                    dict(x=tfno._Strides(-1, 64, 0)), dict(gate=tfno._Strides(1 << 40, 64, 0))):
            assert call(fn, recurrence_desc(**bad), args) == tfno.ERR_SHAPE, bad
        for n in ("x", "gate", "input_gate", "y"):
            assert call(fn, recurrence_desc(**{n: tfno._Strides(0, 1 << 24, 0)}), args) == tfno.ERR_UNSUPPORTED, n
        for n in needed:
            assert call(fn, recurrence_desc(), args, **{n: args[n] + 1}) == tfno.ERR_ALIGN, n
        assert call(fn, recurrence_desc(), args, tape=args["tape"] + 128) == tfno.ERR_ALIGN
        assert call(fn, recurrence_desc(), args, rate=args["rate"] + 2) == tfno.ERR_ALIGN
        out = "y" if "y" in args else "dx"
        for other in ("x", "gate", "input_gate", "rate"):
            assert call(fn, recurrence_desc(), args, **{out: args[other]}) == tfno.ERR_ALIAS, other
        assert call(fn, recurrence_desc(**{out: tfno._Strides(0, 64, 0)}), args) == tfno.ERR_ALIAS           # one place for the whole batch
        assert call(fn, recurrence_desc(**{out: tfno._Strides(512, 32, 0)}), args) == tfno.ERR_ALIAS         # tokens over each other
        assert call(fn, recurrence_desc(B=0), dict.fromkeys(args)) == tfno.OK
    for n, v in (("dinput_gate", None), ("input_gate", None), ("rate", None)):      # a gradient without its input, or the other way
        assert call(L.tfno_gated_recurrence_backward, recurrence_desc(), BACKWARD, **{n: v}) == tfno.ERR_NULL, n
    assert call(L.tfno_gated_recurrence, recurrence_desc(T=0), dict.fromkeys(FORWARD)) == tfno.OK
    assert call(L.tfno_gated_recurrence_backward, recurrence_desc(), BACKWARD, dgate=BACKWARD["dx"]) == tfno.ERR_ALIAS


def test_recurrence_memory(L):
    size = ctypes.byref
    d = recurrence_desc(B=3, T=65, C=10)
    assert L.tfno_gated_recurrence_tape_bytes(size(d)) == 4 * 3 * 3 * 10
    assert L.tfno_gated_recurrence_tape_bytes(None) == 0 and L.tfno_gated_recurrence_tape_bytes(size(recurrence_desc(C=0))) == 0
    many = recurrence_desc(B=4096, T=100, C=64)
    assert L.tfno_gated_recurrence_workspace_bytes(size(many), 0) == 0                  # enough sequences: none in segments
    assert L.tfno_gated_recurrence_workspace_bytes(size(many), 1) >= 4 * 4096 * 64
    long = recurrence_desc(B=1, T=1 << 20, C=8)
    need = L.tfno_gated_recurrence_workspace_bytes(size(long), 0)
    assert 0 < need <= 256 * 12 * 8
    assert L.tfno_set_workspace(None, 0) == tfno.OK
    row = tfno._Strides(8 << 20, 8, 0)
    far = {n: FAKE + i * (1 << 30) for i, n in enumerate(FORWARD)}
    long = recurrence_desc(B=1, T=1 << 20, C=8, **{n: row for n in ("x", "gate", "input_gate", "y")})
    assert call(L.tfno_gated_recurrence, long, far) == tfno.ERR_WORKSPACE
    assert L.tfno_set_workspace(far["x"], need) == tfno.OK                              # a workspace over an input
    assert call(L.tfno_gated_recurrence, long, far) == tfno.ERR_ALIAS
    assert L.tfno_set_workspace(None, 0) == tfno.OK


def test_recurrence_of_a_workgroup_a_cu_goes_without_segments(L):
    """Blocks of 32 channels, of all sequences: with 144 to 256 of them no size is apart from its neighbours."""
    def need(B, C, back=0):
        return L.tfno_gated_recurrence_workspace_bytes(ctypes.byref(recurrence_desc(B=B, T=2048, C=C)), back)

    assert not any(need(B, 20) for B in range(144, 257)) and need(143, 20) > 0
    assert not any(need(4, C) for C in range(36 * 32, 64 * 32 + 1)) and need(4, 35 * 32) > 0
    assert all(need(B, 20, 1) > 12 * 20 * B for B in range(144, 256))                    # the gradient goes in segments there


def test_step_refuses(L):
    args = pointers("x", "gate", "input_gate", "rate", "states", "slots")

    def step(desc, pool=4, y=FAKE + 64 * MB, **kw):
        return L.tfno_gated_recurrence_step(ctypes.byref(desc), *dict(args, **kw).values(), pool, y, None)

    for n in ("x", "gate", "states"):
        assert step(recurrence_desc(T=1), **{n: None}) == tfno.ERR_NULL
    assert step(recurrence_desc(T=2)) == tfno.ERR_SHAPE and step(recurrence_desc(T=1), pool=-1) == tfno.ERR_SHAPE
    assert step(recurrence_desc(T=1), pool=1, slots=None) == tfno.ERR_SHAPE             # fewer states than sequences
    assert step(recurrence_desc(T=1), y=args["x"]) == tfno.ERR_ALIAS and step(recurrence_desc(T=1), y=args["states"]) == tfno.ERR_ALIAS
    assert step(recurrence_desc(T=1), states=args["states"] + 2) == tfno.ERR_ALIGN
    assert step(recurrence_desc(T=1, B=0), pool=0) == tfno.OK


def test_norms_refuse(L, workspace):
    for fn, args, needed in ((L.tfno_block_norm, NORM, ("y", "gate")), (L.tfno_block_norm_backward, NORM_BACK, ("y", "gate", "dy"))):
        assert call(fn, None, args) == tfno.ERR_NULL
        for n in needed:
            assert call(fn, norm_desc(), args, **{n: None}) == tfno.ERR_NULL, n
        for bad in (dict(dtype=2), dict(residual_dtype=2), dict(dtype=0, residual_dtype=1), dict(B=-1), dict(T=-1), dict(C=0), dict(gate_kind=4), dict(gate_kind=-1),
                    dict(activation=3), dict(eps=0.0), dict(eps=math.nan), dict(residual_scale=math.inf), dict(B=1 << 16, T=1 << 15), dict(y=tfno._Strides(-1, 64, 0))):
            assert call(fn, norm_desc(**bad), args) == tfno.ERR_SHAPE, bad
        assert call(fn, norm_desc(C=8193), args) == tfno.ERR_UNSUPPORTED
        for n in needed:
            assert call(fn, norm_desc(), args, **{n: args[n] + 1}) == tfno.ERR_ALIGN, n
        assert call(fn, norm_desc(), args, r=args["r"] + 2) == tfno.ERR_ALIGN           # float32 there
        assert call(fn, norm_desc(B=0, gate_kind=0), dict.fromkeys(args)) == tfno.OK
    both = dict(r_out=None, n_out=None)
    assert call(L.tfno_block_norm, norm_desc(), NORM, **both) == tfno.ERR_NULL
    assert call(L.tfno_block_norm_backward, norm_desc(), NORM_BACK, d_r_out=None, d_n_out=None) == tfno.ERR_NULL
    assert call(L.tfno_block_norm, norm_desc(), NORM, r_out=NORM["n_out"]) == tfno.ERR_ALIAS
    assert call(L.tfno_block_norm, norm_desc(), NORM, r_out=NORM["y"]) == tfno.ERR_ALIAS
    assert call(L.tfno_block_norm, norm_desc(), NORM, r_out=NORM["r"] + 4) == tfno.ERR_ALIAS          # in place, but not at the same place
    assert call(L.tfno_block_norm, norm_desc(), NORM, n_out=NORM["w_before"]) == tfno.ERR_ALIAS
    assert call(L.tfno_block_norm_backward, norm_desc(), NORM_BACK, r=None) == tfno.ERR_NULL          # dr without r
    assert call(L.tfno_block_norm_backward, norm_desc(gate_kind=0), NORM_BACK) == tfno.ERR_NULL       # dgate without a gate
    assert call(L.tfno_block_norm_backward, norm_desc(norm_after=0), NORM_BACK) == tfno.ERR_SHAPE     # the gradient of weights that are not used
    assert call(L.tfno_block_norm_backward, norm_desc(), NORM_BACK, dy=NORM_BACK["dr"]) == tfno.ERR_ALIAS
    assert call(L.tfno_block_norm_backward, norm_desc(), NORM_BACK, dw_after=NORM_BACK["w_after"]) == tfno.ERR_ALIAS
    wide = tfno._Strides(100, 0, 0)
    assert call(L.tfno_block_norm_backward, norm_desc(gate_kind=2, gate=wide, dgate=wide), NORM_BACK) == tfno.ERR_SHAPE
    assert call(L.tfno_block_norm_backward, norm_desc(gate_kind=2, gate=wide, dgate=tfno._Strides(64, 0, 0)), NORM_BACK, dy=None) == tfno.ERR_NULL


def test_norms_need_their_workspace_for_sums_alone(L):
    need = L.tfno_block_norm_workspace_bytes(ctypes.byref(norm_desc()))
    assert need > 0 and L.tfno_block_norm_workspace_bytes(None) == 0 and L.tfno_block_norm_workspace_bytes(ctypes.byref(norm_desc(C=8193))) == 0
    assert L.tfno_set_workspace(None, 0) == tfno.OK
    for n in ("dw_after", "dw_before"):
        assert call(L.tfno_block_norm_backward, norm_desc(), NORM_BACK, **{"dw_after": None, "dw_before": None, n: NORM_BACK[n]}) == tfno.ERR_WORKSPACE
    assert L.tfno_set_workspace(FAKE + 64 * MB, need - 1) == tfno.OK
    assert call(L.tfno_block_norm_backward, norm_desc(), NORM_BACK) == tfno.ERR_WORKSPACE
    assert L.tfno_set_workspace(NORM_BACK["y"], need) == tfno.OK
    assert call(L.tfno_block_norm_backward, norm_desc(), NORM_BACK) == tfno.ERR_ALIAS
    assert L.tfno_set_workspace(None, 0) == tfno.OK


def test_clip_refuses(L, workspace):
    def clip(tensors, limit=1.0, norm=FAKE + 512 * MB):
        array = (tfno._Tensor * max(1, len(tensors)))(*[tfno._Tensor(*t) for t in tensors])
        return L.tfno_clip_grad_norm(ctypes.addressof(array), len(tensors), limit, norm, None)

    one, two = (FAKE, 1000, 0), (FAKE + 4000, 10, 1)
    for limit in (-1.0, math.nan):
        assert clip([one], limit) == tfno.ERR_SHAPE
    assert L.tfno_clip_grad_norm(None, -1, 1.0, None, None) == tfno.ERR_SHAPE
    assert L.tfno_clip_grad_norm(None, 1, 1.0, None, None) == tfno.ERR_NULL
    assert clip([one, (None, 3, 0)]) == tfno.ERR_NULL
    assert clip([(FAKE, -1, 0)]) == tfno.ERR_SHAPE and clip([(FAKE, 1 << 40, 0)]) == tfno.ERR_SHAPE and clip([(FAKE, 1, 2)]) == tfno.ERR_SHAPE
    assert clip([(FAKE + 2, 10, 0)]) == tfno.ERR_ALIGN and clip([(FAKE + 1, 10, 1)]) == tfno.ERR_ALIGN and clip([one], norm=FAKE + 512 * MB + 1) == tfno.ERR_ALIGN
    assert clip([one, one]) == tfno.ERR_ALIAS                                            # the same tensor twice
    assert clip([two, (FAKE, 1001, 0)]) == tfno.ERR_ALIAS                                # the last element of one in another
    assert clip([one, two], norm=FAKE + 400) == tfno.ERR_ALIAS
    assert clip([one, (FAKE + (1 << 32) + 64, 10, 0)]) == tfno.ERR_ALIAS                 # in the workspace
    assert L.tfno_clip_grad_norm_workspace_bytes(-1) == 0
    assert L.tfno_clip_grad_norm_workspace_bytes(1000) > L.tfno_clip_grad_norm_workspace_bytes(1) > 0
    assert L.tfno_set_workspace(FAKE + (1 << 32), L.tfno_clip_grad_norm_workspace_bytes(2) - 1) == tfno.OK
    assert clip([one, two]) == tfno.ERR_WORKSPACE


def test_binding_refuses_what_is_not_on_the_device_or_has_another_type():
    x, f = torch.zeros(2, 8, 64, dtype=torch.bfloat16), torch.zeros(64)
    with pytest.raises(TypeError):
        tfno.gated_recurrence(x, x, x, f, x)                      # on the host
    with pytest.raises(TypeError):
        tfno.gated_recurrence(x.half(), x.half(), None, None, x.half())
    with pytest.raises(TypeError):
        tfno.block_norm(x, x, None, f, f, x, x)
    with pytest.raises(TypeError):
        tfno.gated_recurrence_step(x[:, 0], x[:, 0], None, None, torch.zeros(2, 64), x[:, 0])
    with pytest.raises(TypeError):
        tfno.clip_grad_norm([f], 1.0)
    with pytest.raises(ValueError):
        tfno.block_norm(x, x, None, f, f, x, x, activation="relu")
    assert tfno.clip_grad_norm([], 1.0) is None


@pytest.fixture
def device(monkeypatch):
    """Tensors of the meta device count as ones on a GPU: shapes are checked before anything else is asked of them."""
    def of(t):
        return None if t is None else (t.dtype, 0, t.shape, t.stride())
    monkeypatch.setattr(tfno, "_of", of)
    yield lambda *shape, dtype=torch.float32: torch.empty(*shape, dtype=dtype, device="meta")


def test_binding_refuses_shapes_that_do_not_fit(L, device):
    def recurrence(**kw):
        x = dict(x=device(2, 8, 64), gate=device(2, 8, 64), input_gate=device(2, 8, 64), rate=device(64), y=device(2, 8, 64), dx=None, dgate=None, dinput_gate=None,
                 drate=None, lengths=None, tape=None, initial=None, final=None, other=None)
        x.update(kw)
        return tfno._recurrence_plan(*map(tfno._of, x.values()), True)

    assert recurrence()[1] == 4 * 2 * 64
    for bad in (dict(x=device(8, 64)), dict(gate=device(2, 8, 63)), dict(input_gate=device(1, 8, 64)), dict(rate=device(63)), dict(rate=device(64, 2)[:, 0]),
                dict(y=device(2, 64, 8).transpose(1, 2)), dict(initial=device(2, 63)), dict(final=device(64, 2).t()), dict(lengths=device(3, dtype=torch.int32)),
                dict(tape=device(10, dtype=torch.uint8)), dict(drate=device(1, 64))):
        with pytest.raises(ValueError):
            recurrence(**bad)
    for bad in (dict(gate=device(2, 8, 64, dtype=torch.bfloat16)), dict(rate=device(64, dtype=torch.float64)), dict(lengths=device(2, dtype=torch.int64)),
                dict(initial=device(2, 64, dtype=torch.bfloat16)), dict(tape=device(10000))):
        with pytest.raises(TypeError):
            recurrence(**bad)

    def step(**kw):
        x = dict(x=device(2, 64), gate=device(2, 64), input_gate=None, rate=device(64), y=device(2, 64), states=device(5, 64), slots=None)
        x.update(kw)
        return tfno._recurrence_step_plan(*map(tfno._of, x.values()), True)

    step()
    for bad in (dict(x=device(2, 1, 64)), dict(gate=device(3, 64)), dict(states=device(5, 63)), dict(states=device(64)), dict(slots=device(3, dtype=torch.int32)),
                dict(y=device(64, 2).t())):
        with pytest.raises(ValueError):
            step(**bad)

    def norms(kind=device(2, 8, 64), **kw):
        x = dict(y=device(2, 8, 64), r=device(2, 8, 64), gate=kind, w_after=device(64), w_before=device(64), r_out=device(2, 8, 64), n_out=device(2, 8, 64), dy=None, dr=None,
                 dgate=None, dw_after=None, dw_before=None, lengths=None)
        x.update(kw)
        return tfno._block_norm_plan(*map(tfno._of, x.values()), True, 0, 1.0, 1e-6)

    for kind in (None, device(64), device(2, 64), device(2, 8, 64)):
        assert norms(kind)[1] == 0
        assert norms(kind, dw_after=device(64))[1] > 0
    for bad in (dict(y=device(16, 64)), dict(r=device(2, 8, 63)), dict(kind=device(2, 8, 8, 64)), dict(kind=device(3, 64)), dict(kind=device(63)), dict(w_after=device(63)),
                dict(n_out=device(2, 64, 8).transpose(1, 2)), dict(kind=device(2, 64), dgate=device(64, 2).t()), dict(lengths=device(2, 1, dtype=torch.int32))):
        with pytest.raises(ValueError):
            norms(**bad)
    half = dict(y=device(2, 8, 64, dtype=torch.bfloat16), n_out=device(2, 8, 64, dtype=torch.bfloat16))
    norms(device(64), **half)
    for bad in (dict(kind=device(2, 64, dtype=torch.bfloat16)), dict(half), dict(r=device(2, 8, 64, dtype=torch.bfloat16)),
                dict(half, kind=None, r=device(2, 8, 64, dtype=torch.bfloat16)), dict(w_before=device(64, dtype=torch.bfloat16))):
        with pytest.raises(TypeError):
            norms(**bad)
