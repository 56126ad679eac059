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
