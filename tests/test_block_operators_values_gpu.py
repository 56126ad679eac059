"""The operators of a block along time on the GPU at values where one channel, row or sequence could go wrong beneath the others."""
import math

import pytest
import torch

import block_oracle as oracle
from block_oracle import BF16, F32
from test_block_operators_gpu import (INPUTS, PARTS, TYPES, between_inputs, between_wanted, check_recurrence, empty, near, recur, recur_back, recurrence_inputs,  # noqa: F401
                                      recurrence_wanted, say, tfno)

pytestmark = pytest.mark.gpu


def same_where_finite(name, got, want, bound):
    """Finite where the wanted values are, and as near there as `bound`."""
    finite = torch.isfinite(want)
    assert torch.equal(torch.isfinite(got), finite), f"{name}: {int((torch.isfinite(got) != finite).sum())} values finite in one alone"
    off = oracle.rel(torch.where(finite, got.double(), 0.0), torch.where(finite, want, 0.0))
    say(f"   {name}: {off:.3g} of {bound:.3g}, {int((~finite).sum())} not finite")
    assert off <= bound, name


# ---------------------------------------------------------------- gated linear recurrence

# tokens of a bad gate and of decays of 0: within one group of eight tokens, in either order; in neighbouring groups, in another wave, in another tile; several of each
BAD_AND_RESETS = [([3], [5]), ([5], [3]), ([3], [3]), ([3], [12]), ([12], [3]), ([3], [20]), ([3], [64]), ([3], [130]), ([7], [8]), ([8], [7]), ([0], [1]), ([2, 40], [4, 41, 90])]


def check_bad_gates(tfno, x, bad, resets, value, what, clean=True):
    """`value` in the gates of the tokens `bad` of two channels of three, decays of 0 at the tokens `resets` of one of them and, where `clean`, of the third."""
    say(what)
    dtype, B, T, C = x["x"].dtype, *x["x"].shape
    if x["rate"] is not None:
        x["rate"][:] = x["rate"].clamp(0.05, 2.0)
        x["rate"][0::3] = x["rate"][1::3] = 1000.0              # a gate that is open makes the decay 0, one that is nearly closed leaves something
        x["gate"][:, :, 0::3] -= 7.5
        x["gate"][:, :, 1::3] -= 7.5
    for t in resets:
        for c in (0, 1)[:1 + clean]:
            x["gate"][:, t, c::3] = 90.0 if x["rate"] is not None else -math.inf
    for t in bad:
        x["gate"][:, t, 0::3] = value
        x["gate"][:, t, 2::3] = value
    tape = tfno.gated_recurrence_tape(x["x"])
    y, final = recur(tfno, x, tape)
    w = recurrence_wanted(x)
    same_where_finite("y", y, w[0], oracle.REL[dtype])
    same_where_finite("final", final, w[1], oracle.REL[F32])
    d = recur_back(tfno, x, tape)
    same_where_finite("dx", d["x"], w[2], oracle.REL[dtype])
    for t in resets:                                            # 0 times a gradient that is not finite: either answer will do
        either = ~torch.isfinite(w[2][:, t])
        d["gate"][:, t][either], w[3][:, t][either] = 0.0, 0.0
    same_where_finite("dgate", d["gate"], w[3], oracle.REL_GATES[dtype])
    for n, v in (("input_gate", w[4]), ("rate", w[5])):
        if d[n] is not None:
            same_where_finite("d" + n, d[n], v, oracle.REL_SUMS if n == "rate" else oracle.REL[dtype])
    same_where_finite("dinitial", d["initial"], w[6], oracle.REL[F32])
    return y


@pytest.mark.parametrize("dtype", (F32, BF16))
@pytest.mark.parametrize("gates", ("decay", "decay of inputs", "both", "one"))
@pytest.mark.parametrize("where", range(len(BAD_AND_RESETS)))
def test_recurrence_gates_of_nan_up_to_the_next_reset(tfno, dtype, gates, where):  # noqa: F811
    """A NaN in a gate stays in its channel up to the next decay of 0, forward, and back to the one before, in gradients."""
    bad, resets = BAD_AND_RESETS[where]
    for C, clean in ((7, True), (70, True), (7, False), (70, False)):
        check_bad_gates(tfno, recurrence_inputs(dtype, 2, 150, C, gates, seed=21), bad, resets, math.nan, f"[case] NaN gates {dtype} {gates} {C} {bad} {resets} {clean}", clean)


@pytest.mark.parametrize("dtype", (F32, BF16))
@pytest.mark.parametrize("gates", ("decay", "both"))
def test_recurrence_gates_of_nan_in_segments_and_short_sequences(tfno, dtype, gates):  # noqa: F811
    for size, bad, resets in (((1, 1500, 6), [3], [700]), ((1, 1500, 6), [700], [3]), ((1, 1500, 6), [3, 900], [10, 1200]), ((3, 1100, 40), [500], [520]),
                              ((4200, 13, 70), [2], [5]), ((4200, 30, 70), [2], [17]), ((300, 70, 64), [10], [40])):
        check_bad_gates(tfno, recurrence_inputs(dtype, *size, gates, seed=22), bad, resets, math.nan, f"[case] NaN gates {dtype} {gates} {size} {bad} {resets}")


@pytest.mark.parametrize("where", range(len(BAD_AND_RESETS)))
def test_recurrence_infinite_growth_up_to_the_next_reset(tfno, where):  # noqa: F811
    """A decay of infinity: what comes of it is not finite up to the next decay of 0."""
    bad, resets = BAD_AND_RESETS[where]
    for size in ((2, 150, 7), (1, 1500, 7)):
        check_bad_gates(tfno, recurrence_inputs(F32, *size, "decay", seed=23), bad, resets, math.inf, f"[case] infinite growth {size} {bad} {resets}")


@pytest.mark.parametrize("gates", ("decay", "both"))
def test_recurrence_steps_forget_nans_where_sequences_do(tfno, gates):  # noqa: F811
    x = recurrence_inputs(F32, 2, 40, 7, gates, seed=24)
    y = check_bad_gates(tfno, x, [3, 20], [5, 30], math.nan, f"[case] steps {gates}")
    state = x["initial"].clone()
    for t in range(40):
        o = torch.empty(2, 7, device="cuda")
        one = [None if x[n] is None else x[n] if n == "rate" else x[n][:, t] for n in INPUTS]
        tfno.gated_recurrence_step(*one, state, o, normalise=x["normalise"])
        same_where_finite(f"step {t}", o, y[:, t].double(), oracle.REL[F32])


@pytest.mark.parametrize("dtype", (F32, BF16))
@pytest.mark.parametrize("gates", ("both", "one", "decay", "decay of inputs"))
@pytest.mark.parametrize("size", [(8, 700, 1000), (8, 600, 640), (5, 520, 933), (255, 520, 20), (144, 513, 31), (143, 513, 31), (257, 520, 20), (8, 700, 1030)])
def test_recurrence_of_a_workgroup_a_cu(tfno, dtype, gates, size):  # noqa: F811
    """144 to 256 blocks of 32 channels, for which the forward kernel has its largest workgroups, and the sizes next to them; of different lengths."""
    B, T, C = size
    x = recurrence_inputs(dtype, *size, gates, seed=25)
    x["lengths"] = torch.tensor([T, 0, 1, T - 1, 256, *((b * 101 + 7) % (T + 1) for b in range(5, B))], dtype=torch.int32, device="cuda")
    check_recurrence(tfno, x, f"[case] a workgroup a CU {dtype} {gates} {size}")


def recurrence_sizes(x):
    """What the terms of y, final, and the gradients of x, gate, input_gate, rate and the initial state add up to without their signs.  A float32 result is as far off as its terms'
    roundings, which oracle.REL and the others count for terms of one size, whatever cancels in it.  A decay exp(l) is |l| times as far off as l: l is a product with a sigmoid, which is
    (1 + |gate|) 2^-24 off, and 4 2^-24 more, 10 2^-24 in all; so a term that has gone through decays whose l add up to L has 10 L roundings more.  Each decay counts 1 + |l| / 4 times here:
    their product is 1 + L / 4 at least, and 64 of it the 64 of oracle.REL and 16 L."""
    live = oracle.live_of(x["lengths"], *x["x"].shape[:2], "cuda")
    at, gate, into, d_y = (oracle.only(live, x[n]) for n in ("x", "gate", "input_gate", "d_y"))
    at, d_y = at.abs(), d_y.abs()
    s = None if x["rate"] is None else torch.sigmoid(gate)
    l = gate if s is None else -x["rate"].double() * s
    a, o = l.exp() * (1 - l / 4), torch.ones_like(at) if into is None else torch.sigmoid(into)
    left = torch.sqrt(-torch.expm1(2 * l)) if x["normalise"] else torch.ones_like(at)
    h, before, y = x["initial"].double().abs(), [], torch.zeros_like(at)
    for t in range(at.shape[1]):
        before.append(h)
        h = torch.where(live[:, t], a[:, t] * h + at[:, t] * o[:, t] * left[:, t], h)
        y[:, t] = torch.where(live[:, t], h, 0.0)
    final, D = h, x["d_final"].double().abs()
    dx, dl, do = (torch.zeros_like(at) for _ in range(3))
    for t in reversed(range(at.shape[1])):
        G = D + d_y[:, t]
        through = a[:, t] * before[t]
        if x["normalise"]:
            through = through + at[:, t] * o[:, t] * a[:, t] ** 2 / left[:, t]
        for out, v in ((dx, o[:, t] * left[:, t]), (do, at[:, t] * left[:, t]), (dl, through)):
            out[:, t] = torch.where(live[:, t], G * v, 0.0)
        D = torch.where(live[:, t], a[:, t] * G, D)
    return (y, final, dx, dl if s is None else dl * x["rate"].double() * s * (1 - s), None if into is None else do * o * (1 - o), None if s is None else (dl * s).sum((0, 1)), D)


def near_by_channel(name, got, want, size, bound):
    """Every channel of every sequence by itself (of [B, T, C]), or every value, against the size of its terms."""
    assert torch.isfinite(got).all(), name
    off = got.double() - want
    if got.dim() == 3:
        off, size = off.norm(dim=1), size.norm(dim=1)
    off = off.abs()
    worst = float(torch.where(size > 0, off / size, off).max())
    say(f"   {name}: {worst:.3g} of {bound:.3g} in the worst channel")
    assert worst <= bound, name


@pytest.mark.parametrize("dtype", (F32, BF16))
@pytest.mark.parametrize("gates", ("both", "one", "decay", "decay of inputs"))
@pytest.mark.parametrize("size", [(3, 300, 70), (7, 130, 33), (1, 1500, 6), (5, 513, 933), (4200, 13, 70), (300, 70, 64)])
def test_recurrence_every_channel_by_itself(tfno, dtype, gates, size):  # noqa: F811
    """Channels and sequences whose values, gradients and rates differ by orders of magnitude, and sequences of few tokens among long ones."""
    B, T, C = size
    x = recurrence_inputs(dtype, *size, gates, seed=26)
    gen = torch.Generator("cuda").manual_seed(26)

    def scales(*shape):
        return 10.0 ** (6 * torch.rand(*shape, generator=gen, device="cuda") - 3)

    for values, state in (("x", "initial"), ("d_y", "d_final")):
        scale = scales(B, C)
        x[values], x[state] = (x[values].float() * scale[:, None]).to(dtype), x[state] * scale
    if x["rate"] is not None:
        x["rate"] = 10.0 ** (7 * torch.rand(C, generator=gen, device="cuda") - 5)
    if B > 1:
        x["lengths"] = torch.tensor([T, 1, *(1 + (b * 101 + 7) % T for b in range(2, B))], dtype=torch.int32, device="cuda")
    say(f"[case] channels {dtype} {gates} {size}")
    tape = tfno.gated_recurrence_tape(x["x"])
    y, final = recur(tfno, x, tape)
    d = recur_back(tfno, x, tape)
    bounds = (oracle.REL[dtype], oracle.REL[F32], oracle.REL[dtype], oracle.REL_GATES[dtype], oracle.REL[dtype], oracle.REL_SUMS, oracle.REL[F32])
    for n, got, w, s, bound in zip(("y", "final", "dx", "dgate", "dinput", "drate", "dinitial"), (y, final, *(d[k] for k in (*INPUTS, "initial"))), recurrence_wanted(x),
                                   recurrence_sizes(x), bounds):
        if got is not None:
            near_by_channel(n, got, w, s, bound)


# ---------------------------------------------------------------- norms around a block

def norms_and_gradients(tfno, x):
    out = [empty(x["y"], x["d_r"].dtype), empty(x["y"])]
    tfno.block_norm(*(x[n] for n in PARTS), *out, **x["ways"])
    d = [empty(x[n]) for n in PARTS]
    tfno.block_norm_backward(*(x[n] for n in PARTS), x["d_r"], x["d_n"], *d, **x["ways"])
    return dict(zip(("r_out", "n_out", *("d" + n for n in PARTS)), (*out, *d)))


def bound_of(name, t):
    if name in ("r_out", "n_out"):
        return oracle.REL[t.dtype]
    return oracle.REL_GATES[BF16] if t.dtype == BF16 else oracle.REL_SUMS


@pytest.mark.parametrize("types", TYPES)
@pytest.mark.parametrize("activation", ("none", "silu", "sigmoid"))
@pytest.mark.parametrize("size", [(6, 50, 40), (6, 50, 100), (5, 33, 1024), (4, 7, 5000), (300, 3, 40), (70, 40, 256), (3, 1300, 64)])
def test_norms_gates_of_sequences_without_tokens(tfno, types, activation, size):  # noqa: F811
    """The gate of a sequence of no tokens counts in no sum, whatever it is."""
    B, T, C = size
    x = between_inputs(*types, *size, "sequence", activation, seed=21)
    lengths = [(b * 7 + 2) % (T + 1) for b in range(B)]
    lengths[0], lengths[1], lengths[-1] = T, 0, -1
    x["ways"]["lengths"] = torch.tensor(lengths, dtype=torch.int32, device="cuda")
    none = x["ways"]["lengths"] <= 0
    x["gate"][none] = 0.0
    w = dict(zip(("r_out", "n_out", *("d" + n for n in PARTS)), between_wanted(x)))
    for bad in (math.nan, math.inf, -math.inf):
        say(f"[case] gates of nothing {types} {activation} {size} {bad}")
        x["gate"][none] = bad
        for n, got in norms_and_gradients(tfno, x).items():
            near(n, got, w[n], bound_of(n, got))
            if n == "dgate":
                assert (got[none] == 0).all()


@pytest.mark.parametrize("gate", ("token", "sequence", "channel"))
@pytest.mark.parametrize("C", (40, 1024))
def test_norms_of_no_tokens_at_all_have_sums_of_zero(tfno, gate, C):  # noqa: F811
    x = between_inputs(F32, F32, 4, 9, C, gate, "silu", seed=22)
    x["ways"]["lengths"] = torch.zeros(4, dtype=torch.int32, device="cuda")
    for n in ("y", "r", "gate", "w_after", "w_before", "d_r", "d_n"):
        x[n].fill_(math.nan)
    for n, got in norms_and_gradients(tfno, x).items():
        assert (got == 0).all(), n


def near_by_row(name, got, want, bound):
    """Every row by itself: got and want are [..., C]."""
    assert torch.isfinite(got).all(), name
    off, size = (got.double() - want).norm(dim=-1), want.norm(dim=-1)
    worst = float(torch.where(size > 0, off / size, off).max())
    say(f"   {name}: {worst:.3g} of {bound:.3g} in the worst row")
    assert worst <= bound, name


@pytest.mark.parametrize("types", TYPES)
@pytest.mark.parametrize("after", (True, False))
@pytest.mark.parametrize("C", (40, 205, 1024, 4099))
def test_norms_and_gradient_of_rows_of_any_size(tfno, types, after, C):  # noqa: F811
    """Rows from 1e-15 to 1e17, whose inverse roots' third powers are far out of float32's range, and of zeros; the squares' sums are not."""
    sizes = torch.tensor([1e-15, 1e-10, 1e-5, 1.0, 1e5, 1e10, 1e13, 1e15, 1e17, 0.0], device="cuda")
    x = between_inputs(*types, 2, len(sizes), C, "token", "silu", seed=23, after=after)
    gen = torch.Generator("cuda").manual_seed(23)
    for n in ("y", "r"):
        x[n] = (torch.randn(2, len(sizes), C, generator=gen, device="cuda") * sizes[:, None]).to(x[n].dtype)
    x["ways"]["eps"] = 1e-30
    say(f"[case] sizes of rows {types} {after} {C}")
    out, d = [empty(x["y"], types[1]), empty(x["y"])], [empty(x[n]) for n in PARTS]
    tfno.block_norm(*(x[n] for n in PARTS), *out, **x["ways"])
    if not after:
        d[3] = None
    tfno.block_norm_backward(*(x[n] for n in PARTS), x["d_r"], x["d_n"], *d, **x["ways"])
    w = between_wanted(x)
    for n, got, want in zip(("r_out", "n_out", "dy", "dr", "dgate"), (*out, *d), w):
        near_by_row(n, got, want, bound_of(n, got))
    for got in d[3:]:
        assert got is None or torch.isfinite(got).all()


def sums_sizes(x):
    """What the terms of dw_after, dw_before and of the gradient of a gate that tokens share add up to without their signs; the two terms of the slope of z sigmoid(z), which cancel near
    z = -1.28, among them."""
    w = x["ways"]
    live = oracle.live_of(w["lengths"], *x["y"].shape[:2], "cuda")
    y, r, d_r, d_n = (oracle.only(live, x[n]) for n in ("y", "r", "d_r", "d_n"))
    wa, wb, gate = (None if x[n] is None else x[n].double() for n in ("w_after", "w_before", "gate"))
    m = y / torch.sqrt((y * y).mean(-1, keepdim=True) + w["eps"])
    z, slope = torch.ones_like(m), torch.zeros_like(m)
    if gate is not None:
        g = oracle.only(live, gate) if gate.dim() == 3 else gate[:, None].expand_as(m) if gate.dim() == 2 else gate.expand_as(m)
        o = torch.sigmoid(g)
        z, slope = {"none": (g, torch.ones_like(g)), "silu": (g * o, o * (1 + g.abs() * (1 - o))), "sigmoid": (o, o * (1 - o))}[w["activation"]]
    stream, size = w["residual_scale"] * r + z * m * wa, (w["residual_scale"] * r).abs() + (z * m * wa).abs()
    q = 1 / torch.sqrt((stream * stream).mean(-1, keepdim=True) + w["eps"])
    b = (d_n * wb).abs()
    d = d_r.abs() + q * (b + size * q * (q * (b * size).mean(-1, keepdim=True)))
    of_gate = torch.where(live, d * (m * wa * slope).abs(), 0.0)
    return (d * (z * m).abs()).sum((0, 1)), (d_n.abs() * size * q).sum((0, 1)), of_gate.sum(1) if gate is not None and gate.dim() == 2 else of_gate.sum((0, 1))


@pytest.mark.parametrize("types", TYPES)
@pytest.mark.parametrize("gate", ("none", "token", "sequence", "channel"))
@pytest.mark.parametrize("size", [(2, 30, 40), (3, 700, 64), (900, 5, 40), (2100, 70, 64), (600, 20, 256), (70, 40, 1000), (9, 6, 5000)])
def test_norms_every_row_and_channel_by_itself(tfno, types, gate, size):  # noqa: F811
    """Rows whose values and gradients differ by orders of magnitude; many sequences with gates of their own, long and short ones."""
    B, T, C = size
    x = between_inputs(*types, *size, gate, "silu", seed=24)
    gen = torch.Generator("cuda").manual_seed(24)
    for names in (("y",), ("r",), ("d_r", "d_n")):
        scale = 10.0 ** (4 * torch.rand(B, T, 1, generator=gen, device="cuda") - 2)
        for n in names:
            x[n] = (x[n].float() * scale).to(x[n].dtype)
    x["ways"]["lengths"] = torch.tensor([T, *(1 + (b * 101 + 7) % T for b in range(1, B))], dtype=torch.int32, device="cuda")
    say(f"[case] rows by themselves {types} {gate} {size}")
    got, w = norms_and_gradients(tfno, x), between_wanted(x)
    sizes = dict(zip(("dw_after", "dw_before", "dgate"), sums_sizes(x)))
    for (n, t), want in zip(got.items(), w):
        if t is None:
            continue
        if t.dim() == 3:
            near_by_row(n, t, want, bound_of(n, t))
        else:
            near_by_channel(n, t, want, sizes[n], oracle.REL_SUMS)


# ---------------------------------------------------------------- clipping

def test_clip_skips_parameters_without_a_gradient(tfno):  # noqa: F811
    """As a list of parameters' gradients has them: None where a weight is frozen or was not used."""
    model = torch.nn.Sequential(torch.nn.Linear(30, 40), torch.nn.Linear(40, 50), torch.nn.Linear(50, 3)).cuda()
    model[0].weight.requires_grad_(False)
    model[1](torch.randn(7, 40, device="cuda")).square().sum().backward()
    grads, norm = [p.grad for p in model.parameters()], torch.empty((), device="cuda")
    assert grads[0] is None and grads[-1] is None
    want = math.sqrt(sum(float(g.double().square().sum()) for g in grads if g is not None))
    scaled = [g.double() * (0.5 / want) for g in grads if g is not None]
    tfno.clip_grad_norm((p.grad for p in model.parameters()), 0.5, norm)
    assert abs(float(norm) - want) <= 2.0 ** -23 * want
    for g, w in zip((g for g in grads if g is not None), scaled):
        near("clipped", g, w, 2.0 ** -24 * (1 + 2.0 ** -10))
    tfno.clip_grad_norm(grads, 0.25)                            # a device to go by without a norm
    near("clipped again", grads[2], scaled[0] / 2, 2.0 ** -23 * (1 + 2.0 ** -10))
    tfno.clip_grad_norm([None, None], 1.0, norm)
    assert float(norm) == 0 and tfno.clip_grad_norm([None], 1.0) is None
    with pytest.raises(TypeError):
        tfno.clip_grad_norm([None, grads[2], 3.0], 1.0)


@pytest.mark.parametrize("million", (70, 90))
def test_clip_of_what_caches_hold_and_of_more(tfno, million):  # noqa: F811
    """280 and 360 MB: both ways to load and store, whole pieces and their ends."""
    n = million * 1000 * 1000
    gen = torch.Generator("cuda").manual_seed(million)
    memory = torch.randn(n // 2 + 5, generator=gen, device="cuda")
    tensors = [memory[1:n // 2 + 1], torch.randn(n + 3, generator=gen, device="cuda").to(BF16)[3:], torch.randn(7, generator=gen, device="cuda")]
    before, norm = [t.clone() for t in tensors], torch.empty((), device="cuda")
    ends = memory[[0, -4, -3, -2, -1]].clone()
    want = math.sqrt(sum(float(t.double().square().sum()) for t in tensors))
    tfno.clip_grad_norm(tensors, math.inf, norm)
    assert abs(float(norm) - want) <= 2.0 ** -23 * want and all(torch.equal(a, b) for a, b in zip(tensors, before))
    tfno.clip_grad_norm(tensors, 1.0, norm)
    assert abs(float(norm) - want) <= 2.0 ** -23 * want and torch.equal(memory[[0, -4, -3, -2, -1]], ends)
    for t, b in zip(tensors, before):
        near(str(t.dtype), t, b.double() / want, (2.0 ** -8 if t.dtype == BF16 else 2.0 ** -24) * (1 + 2.0 ** -10))
