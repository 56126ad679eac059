"""The gated linear recurrence, the norms around a block and the clipping of gradients on the GPU against float64."""
import math

import pytest
import torch

import block_oracle as oracle
from block_oracle import BF16, F32

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def tfno():
    from paper_2504_11681_amd import binding
    assert torch.cuda.is_available(), "these tests need the MI355X"
    binding.lib()
    return binding


def say(*a):
    print(*a, flush=True)


def near(name, got, want, bound):
    off = oracle.rel(got, want)
    say(f"   {name}: {off:.3g} of {bound:.3g}")
    assert off <= bound, name


def empty(t, dtype=None):
    return None if t is None else torch.full(t.shape, 7.0, dtype=dtype or t.dtype, device="cuda")


# ---------------------------------------------------------------- gated linear recurrence

GATES = ("both", "one", "decay", "decay of inputs")


def recurrence_inputs(dtype, B, T, C, gates="both", seed=0, state=True):
    gen = torch.Generator("cuda").manual_seed(100 + seed)

    def normal(*shape):
        return torch.randn(*shape, generator=gen, device="cuda")

    x = {"x": normal(B, T, C).to(dtype), "input_gate": None, "rate": None, "normalise": gates in ("both", "one"), "lengths": None,
         "initial": normal(B, C) if state else None}
    if gates.startswith("decay"):
        x["gate"] = (-torch.rand(B, T, C, generator=gen, device="cuda") * torch.exp(normal(C) - 2)).to(dtype)
        if gates == "decay of inputs":
            x["input_gate"], x["normalise"] = normal(B, T, C).to(dtype), True
    else:
        x["gate"], x["rate"] = normal(B, T, C).to(dtype), torch.exp(2 * normal(C) - 2)
        if gates == "both":
            x["input_gate"] = normal(B, T, C).to(dtype)
    x["d_y"], x["d_final"] = normal(B, T, C).to(dtype), normal(B, C)
    return x


INPUTS = ("x", "gate", "input_gate", "rate")


def recur(tfno, x, tape=None, y=None):
    y = empty(x["x"]) if y is None else y
    final = torch.full((x["x"].shape[0], x["x"].shape[2]), 7.0, device="cuda")
    tfno.gated_recurrence(*(x[n] for n in INPUTS), y, normalise=x["normalise"], initial_state=x["initial"], final_state=final, lengths=x["lengths"], tape=tape)
    return y, final


def recur_back(tfno, x, tape, grads=None):
    d = grads or {n: empty(x[n]) for n in INPUTS}
    d["initial"] = torch.full((x["x"].shape[0], x["x"].shape[2]), 7.0, device="cuda")
    tfno.gated_recurrence_backward(*(x[n] for n in INPUTS), x["d_y"], *(d[n] for n in INPUTS), tape, normalise=x["normalise"], d_final_state=x["d_final"],
                                   d_initial_state=d["initial"], lengths=x["lengths"])
    return d


def recurrence_wanted(x, grads=True):
    return oracle.recurrence(*(x[n] for n in INPUTS), x["normalise"], x["initial"], x["lengths"], *((x["d_y"], x["d_final"]) if grads else ()))


def check_recurrence(tfno, x, what):
    say(what)
    dtype = x["x"].dtype
    y, final = recur(tfno, x)
    w = recurrence_wanted(x)
    near("y", y, w[0], oracle.REL[dtype])
    near("final", final, w[1], oracle.REL[F32])
    tape = tfno.gated_recurrence_tape(x["x"])
    y2, final2 = recur(tfno, x, tape)
    assert torch.equal(y2, y) and torch.equal(final2, final)
    d = recur_back(tfno, x, tape)
    near("dx", d["x"], w[2], oracle.REL[dtype])
    near("dgate", d["gate"], w[3], oracle.REL_GATES[dtype])
    for n, v in (("input_gate", w[4]), ("rate", w[5])):
        if d[n] is not None:
            near("d" + n, d[n], v, oracle.REL_SUMS if n == "rate" else oracle.REL[dtype])
    near("dinitial", d["initial"], w[6], oracle.REL[F32])
    return y, final, d


# one token and one channel, around the sizes of tiles and of what the tape holds, odd and even channels, several blocks of them
SIZES = [(1, 1, 1), (3, 2, 2), (2, 7, 5), (1, 31, 64), (2, 32, 128), (2, 33, 130), (1, 63, 16), (3, 64, 33), (2, 65, 200), (4, 127, 31), (1, 129, 512), (2, 257, 65)]


@pytest.mark.parametrize("dtype", (F32, BF16))
@pytest.mark.parametrize("gates", GATES)
@pytest.mark.parametrize("size", SIZES)
def test_recurrence_and_gradient(tfno, dtype, gates, size):
    check_recurrence(tfno, recurrence_inputs(dtype, *size, gates), f"[case] recurrence {dtype} {gates} {size}")


@pytest.mark.parametrize("dtype", (F32, BF16))
@pytest.mark.parametrize("size", [(1, 2000, 8), (1, 1025, 96), (2, 1100, 7), (40, 130, 256), (9, 300, 1000), (300, 70, 64)])
def test_recurrence_of_long_sequences_and_many_channels(tfno, dtype, size):
    """Few channels of long sequences, which go in segments, and many."""
    for gates in ("both", "decay"):
        check_recurrence(tfno, recurrence_inputs(dtype, *size, gates, seed=1), f"[case] long {dtype} {gates} {size}")


@pytest.mark.parametrize("dtype", (F32, BF16))
@pytest.mark.parametrize("size", [(3000, 5, 9), (4200, 13, 70), (2100, 30, 64), (1, 9000, 3)])
def test_recurrence_of_many_short_sequences_and_of_a_very_long_one(tfno, dtype, size):
    """So many sequences that each is one wave's, and that their parts of the rates' gradient are added up in pieces; so long a one that it goes in more than a hundred segments."""
    for gates in ("both", "one") if size[0] > 1 else ("both",):
        check_recurrence(tfno, recurrence_inputs(dtype, *size, gates, seed=13), f"[case] many {dtype} {gates} {size}")


@pytest.mark.parametrize("dtype", (F32, BF16))
@pytest.mark.parametrize("T", (100, 1100))
def test_recurrence_of_strong_decays(tfno, dtype, T):
    """Products of decays that underflow within a few tokens, without a decay of 0 among them; then some of those too."""
    x = recurrence_inputs(dtype, 2, T, 20, "decay", seed=14)
    gen = torch.Generator("cuda").manual_seed(14)
    x["gate"] = (-40.0 * torch.rand(2, T, 20, generator=gen, device="cuda") ** 3).to(dtype)
    x["gate"][:, ::7, ::3] = -95.0
    check_recurrence(tfno, x, f"[case] strong {dtype} {T}")
    x["gate"][:, 3::11, 1::4] = -120.0
    x["gate"][:, 5::13, 2::4] = -math.inf
    check_recurrence(tfno, x, f"[case] strong with resets {dtype} {T}")


@pytest.mark.parametrize("dtype", (F32, BF16))
@pytest.mark.parametrize("T", (70, 700, 1500))
def test_recurrence_lengths_and_what_stands_past_them(tfno, dtype, T):
    x = recurrence_inputs(dtype, 8, T, 24, seed=2)
    x["lengths"] = torch.tensor([T, 0, 1, T // 2, 32, T + 50, -3, T - 1], dtype=torch.int32, device="cuda")
    live = oracle.live_of(x["lengths"], 8, T, "cuda")[..., 0]
    for n in ("x", "gate", "input_gate", "d_y"):
        x[n][~live] = float("nan")
    y, final, d = check_recurrence(tfno, x, f"[case] lengths {dtype} {T}")
    for t in (y, d["x"], d["gate"], d["input_gate"]):
        assert (t[~live] == 0).all()
    assert torch.equal(final[1], x["initial"][1]) and torch.equal(d["initial"][1], x["d_final"][1])


@pytest.mark.parametrize("dtype", (F32, BF16))
@pytest.mark.parametrize("T", (90, 1200))
def test_recurrence_resets_and_nans(tfno, dtype, T):
    """Decays of 0 forget what was, NaN too; a NaN stays in its channel up to the next of them; the gradient does not cross them."""
    x = recurrence_inputs(dtype, 2, T, 6, "decay", seed=3)
    resets = [0, 37, 64, T - 2]
    for t in resets:
        x["gate"][:, t, :3] = -math.inf
    check_recurrence(tfno, x, f"[case] resets {dtype} {T}")
    clean, _ = recur(tfno, x)
    x["x"][:, 20, 0] = float("nan")
    x["initial"][:, 1] = float("nan")
    x["initial"][:, 4] = float("nan")
    x["x"][:, 40, 5] = math.inf
    x["gate"][:, 50:60, 4] = -90.0                   # a product of decays that underflows is no decay of 0
    tape = tfno.gated_recurrence_tape(x["x"])
    y, final = recur(tfno, x, tape)
    assert torch.isnan(y[:, 20:37, 0]).all() and torch.equal(y[:, :20, 0], clean[:, :20, 0]) and torch.equal(y[:, 37:, 0], clean[:, 37:, 0])
    assert torch.equal(y[:, :, 1:4], clean[:, :, 1:4])
    assert torch.isnan(y[:, :, 4]).all() and torch.isnan(final[:, 4]).all()
    assert not torch.isfinite(y[:, 40:, 5]).any() and torch.equal(y[:, :40, 5], clean[:, :40, 5])
    d = recur_back(tfno, x, tape)
    assert torch.isfinite(d["x"][:, :, 1:4]).all() and torch.isfinite(d["gate"][:, :, 1:4]).all()
    for t in resets:
        assert (d["gate"][:, t, 1:3] == 0).all()
    assert (d["initial"][:, :3] == 0).all()


def test_recurrence_remembers_for_long(tfno):
    """Decays of 1 - 1e-5 and less: as far off as any other, though 1 minus a float32 decay itself is off by 1e-3 there."""
    x = recurrence_inputs(F32, 2, 2000, 40, "decay", seed=4)
    x["gate"] = -10.0 ** torch.linspace(-7, -4, 40, device="cuda").expand(2, 2000, 40).contiguous()
    x["x"] = x["x"] * 0.01 + 1
    check_recurrence(tfno, x, "[case] long memory")
    x["normalise"] = True
    check_recurrence(tfno, x, "[case] long memory, normalised")


@pytest.mark.parametrize("dtype", (F32, BF16))
def test_recurrence_gates_at_their_ends(tfno, dtype):
    """Gates far open and far closed, rates of 0 and large ones, no decay at all."""
    x = recurrence_inputs(dtype, 2, 150, 12, "both", seed=5)
    x["gate"][:, ::3] = 90.0
    x["gate"][:, 1::3] = -90.0
    x["input_gate"][:, ::4] = 200.0
    x["input_gate"][:, 1::4] = -200.0
    x["rate"][::4] = 0.0
    x["rate"][1::4] = 300.0
    y, final, d = check_recurrence(tfno, x, f"[case] ends {dtype}")
    x = recurrence_inputs(dtype, 2, 150, 12, "decay", seed=6)
    x["gate"].zero_()
    check_recurrence(tfno, x, f"[case] no decay {dtype}")


@pytest.mark.parametrize("dtype", (F32, BF16))
@pytest.mark.parametrize("way", ("fused", "tokens first", "one element off", "repeated", "odd rows"))
def test_recurrence_strides(tfno, dtype, way):
    B, T, C = 3, 77, 24
    x = recurrence_inputs(dtype, B, T, C, seed=7)
    names = ("x", "gate", "input_gate", "d_y")
    grads = {n: empty(x[n]) for n in INPUTS}
    y = None
    if way == "fused":
        w = torch.empty(B, T, 4 * C, dtype=dtype, device="cuda")
        dw = torch.empty_like(w)
        for n, p, dp in zip(("x", "gate", "input_gate"), w.split(C, -1), dw.split(C, -1)):
            x[n], grads[n] = p.copy_(x[n]), dp
        y = w[..., 3 * C:]
    elif way == "tokens first":
        for n in names:
            x[n] = x[n].transpose(0, 1).contiguous().transpose(0, 1)
        grads["x"] = torch.empty(T, B, C, dtype=dtype, device="cuda").transpose(0, 1)
    elif way == "one element off":
        x["gate"] = torch.empty(B * T * C + 1, dtype=dtype, device="cuda")[1:].view(B, T, C).copy_(x["gate"])
    elif way == "repeated":
        x["gate"] = x["gate"][:, :1].expand(-1, T, -1)
        x["input_gate"] = x["input_gate"][:1].expand(B, -1, -1)
    else:
        for n in names:
            x[n] = torch.full((B, T, C + 3), float("nan"), dtype=dtype, device="cuda")[..., :C].copy_(x[n])
    say(f"[case] strides {dtype} {way}")
    tape = tfno.gated_recurrence_tape(x["x"])
    y, final = recur(tfno, x, tape, y)
    d = recur_back(tfno, x, tape, grads)
    w = recurrence_wanted(x)
    near("y", y, w[0], oracle.REL[dtype])
    near("final", final, w[1], oracle.REL[F32])
    for n, v in zip(INPUTS, w[2:6]):
        near("d" + n, d[n], v, oracle.REL_SUMS if n == "rate" else oracle.REL_GATES[dtype])


def test_recurrence_of_nothing(tfno):
    state = torch.randn(3, 5, device="cuda")
    x = torch.empty(3, 0, 5, device="cuda")
    final, d_initial, drate = torch.empty_like(state), torch.empty_like(state), torch.full((5,), 7.0, device="cuda")
    rate = torch.ones(5, device="cuda")
    tape = tfno.gated_recurrence_tape(x)
    tfno.gated_recurrence(x, x, None, rate, torch.empty_like(x), initial_state=state, final_state=final, tape=tape)
    tfno.gated_recurrence_backward(x, x, None, rate, x.clone(), x.clone(), x.clone(), None, drate, tape, d_final_state=state, d_initial_state=d_initial)
    assert torch.equal(final, state) and torch.equal(d_initial, state) and (drate == 0).all()
    none, drate = torch.empty(0, 4, 5, device="cuda"), torch.full((5,), 7.0, device="cuda")
    tfno.gated_recurrence(none, none, None, rate, none.clone())
    tfno.gated_recurrence_backward(none, none, None, rate, none.clone(), none.clone(), none.clone(), None, drate, torch.empty(0, dtype=torch.uint8, device="cuda"))
    assert (drate == 0).all()


def test_recurrence_offsets_past_32_bits(tfno):
    far, T, C = 2 ** 31 + 64, 70, 64
    memory = torch.empty(far + 2 * T * C, dtype=BF16, device="cuda")
    x = recurrence_inputs(BF16, 2, T, C, seed=8)
    x["x"] = memory.as_strided((2, T, C), (far, C, 1)).copy_(x["x"])
    y = memory[T * C:].as_strided((2, T, C), (far, C, 1))
    say("[case] far")
    y, _ = recur(tfno, x, None, y)
    near("y", y, recurrence_wanted(x, False)[0], oracle.REL[BF16])


def test_recurrence_gradient_against_differences(tfno):
    """Central differences of the loss along one direction for each input, at two steps, joined so that what is left of third order in the step cancels.  The loss is
    a sum of products taken in float64 from states that are 2^-24 off each; over a change of 1e-3 of itself that is 1e-3 at most."""
    x = recurrence_inputs(F32, 2, 90, 10, seed=9)
    tape = tfno.gated_recurrence_tape(x["x"])
    recur(tfno, x, tape)
    d = recur_back(tfno, x, tape)

    def loss(x):
        y, final = recur(tfno, x)
        return float((y.double() * x["d_y"].double()).sum() + (final.double() * x["d_final"].double()).sum())

    for n in (*INPUTS, "initial"):
        g = d[n].double()
        if n == "rate":                     # by its logarithm: a rate is not negative
            g = g * x[n].double()
            step = (g / g.norm() * 0.02 * 10 ** 0.5).float()
            moved = [x[n] * torch.exp(h * step) for h in (1.0, -1.0, 0.5, -0.5)]
        else:
            step = (g / g.norm() * (0.02 * float(x[n].norm()))).float()
            moved = [x[n] + h * step for h in (1.0, -1.0, 0.5, -0.5)]
        at = [loss(dict(x, **{n: v})) for v in moved]
        slopes = [(at[0] - at[1]) / 2, at[2] - at[3]]
        slope, want = (4 * slopes[1] - slopes[0]) / 3, float((g * step.double()).sum())
        say(n, slope, want)
        assert abs(slope - want) <= 1e-2 * abs(want), n


@pytest.mark.parametrize("dtype", (F32, BF16))
def test_recurrence_equal_calls_give_equal_bits_and_the_past_does_not_see_the_future(tfno, dtype):
    x = recurrence_inputs(dtype, 2, 1100, 12, seed=10)
    tape = tfno.gated_recurrence_tape(x["x"])
    first, d = recur(tfno, x, tape), recur_back(tfno, x, tape)
    again, d2 = recur(tfno, x, tape), recur_back(tfno, x, tape)
    assert all(torch.equal(a, b) for a, b in zip(first, again))
    assert all(torch.equal(d[n], d2[n]) for n in d)
    other = dict(x, x=x["x"].clone())
    other["x"][:, 600:] = 3.0
    assert torch.equal(recur(tfno, other)[0][:, :600], first[0][:, :600])


@pytest.mark.parametrize("dtype", (F32, BF16))
@pytest.mark.parametrize("gates", GATES)
@pytest.mark.parametrize("size", [(1, 1), (3, 64), (5, 77), (200, 512), (2, 1500)])
def test_recurrence_step(tfno, dtype, gates, size):
    B, C = size
    x = recurrence_inputs(dtype, B, 1, C, gates, seed=11)
    pool = B + 3
    states = torch.randn(pool, C, device="cuda")
    slots = torch.randperm(pool, device="cuda")[:B].to(torch.int32)
    if B > 2:
        slots[1] = -1
        slots[2] = pool
    x["initial"] = states[slots.clamp(0, pool - 1).long()]
    w = recurrence_wanted(x, False)
    before = states.clone()
    one = {n: None if x[n] is None else x[n] if n == "rate" else x[n][:, 0] for n in INPUTS}
    y = torch.full((B, C), 7.0, dtype=dtype, device="cuda")
    tfno.gated_recurrence_step(*(one[n] for n in INPUTS), states, y, normalise=x["normalise"], slots=slots)
    say(f"[case] step {dtype} {gates} {size}")
    there = [b for b in range(B) if not (B > 2 and b in (1, 2))]
    near("y", y[there], w[0][there, 0], oracle.REL[dtype])
    near("states", states[slots[there].long()], w[1][there], oracle.REL[F32])
    untouched = [i for i in range(pool) if i not in {int(slots[b]) for b in there}]
    assert torch.equal(states[untouched], before[untouched])
    if B > 2:
        assert (y[1] == 0).all() and torch.isnan(y[2]).all()


@pytest.mark.parametrize("dtype", (F32, BF16))
def test_recurrence_steps_follow_the_whole_sequence(tfno, dtype):
    x = recurrence_inputs(dtype, 3, 80, 20, seed=12)
    y, final = recur(tfno, x)
    state = x["initial"].clone()
    for t in range(80):
        o = torch.empty(3, 20, dtype=dtype, device="cuda")
        tfno.gated_recurrence_step(x["x"][:, t], x["gate"][:, t], x["input_gate"][:, t], x["rate"], state, o, normalise=True)
        assert oracle.rel(o, y[:, t].double()) <= oracle.REL[dtype]
    near("final", state, final.double(), oracle.REL[F32])


# ---------------------------------------------------------------- norms around a block

def between_inputs(dtype, residual, B, T, C, gate="token", activation="none", seed=0, after=True):
    gen = torch.Generator("cuda").manual_seed(200 + seed)

    def normal(*shape):
        return torch.randn(*shape, generator=gen, device="cuda")

    shapes = {"none": None, "token": (B, T, C), "sequence": (B, C), "channel": (C,)}
    x = {"y": (normal(B, T, C) * torch.exp(normal(B, T, 1))).to(dtype), "r": None if residual is None else normal(B, T, C).to(residual),
         "gate": None if gate == "none" else normal(*shapes[gate]).to(dtype if gate == "token" else F32), "w_after": 1 + 0.2 * normal(C), "w_before": 1 + 0.2 * normal(C)}
    x["d_r"], x["d_n"] = normal(B, T, C).to(residual or dtype), normal(B, T, C).to(dtype)
    x["ways"] = {"norm_after": after, "activation": activation, "residual_scale": 0.75, "eps": 1e-5, "lengths": None}
    return x


PARTS = ("y", "r", "gate", "w_after", "w_before")


def between_wanted(x, d_r=True, d_n=True):
    w = x["ways"]
    return oracle.between(*(x[n] for n in PARTS), w["norm_after"], w["activation"], w["residual_scale"], w["eps"], w["lengths"], x["d_r"] if d_r else None,
                          x["d_n"] if d_n else None)


def check_between(tfno, x, what, which=(True, True)):
    say(what)
    y, dtype, res = x["y"], x["y"].dtype, x["d_r"].dtype
    out = [empty(y, res) if which[0] else None, empty(y) if which[1] else None]
    tfno.block_norm(*(x[n] for n in PARTS), *out, **x["ways"])
    w = between_wanted(x, *which)
    for n, got, want in zip(("r_out", "n_out"), out, w):
        if got is not None:
            near(n, got, want, oracle.REL[got.dtype])
    d = [empty(x[n]) for n in PARTS]
    if not x["ways"]["norm_after"]:
        d[3] = None
    tfno.block_norm_backward(*(x[n] for n in PARTS), x["d_r"] if which[0] else None, x["d_n"] if which[1] else None, *d, **x["ways"])
    for n, got, want in zip(PARTS, d, w[2:]):
        if got is not None:
            want = torch.zeros_like(got, dtype=torch.float64) if want is None else want
            near("d" + n, got, want, oracle.REL_GATES[BF16] if got.dtype == BF16 else oracle.REL_SUMS)
    return out, d


TYPES = ((F32, F32), (BF16, F32), (BF16, BF16))
WIDTHS = [(1, 1, 1), (2, 3, 2), (3, 5, 7), (2, 9, 8), (2, 17, 64), (1, 33, 65), (3, 40, 128), (2, 21, 205), (2, 10, 512), (3, 7, 520), (2, 6, 1000), (2, 5, 2048), (1, 9, 4096),
          (2, 3, 4099), (1, 5, 8192)]


@pytest.mark.parametrize("types", TYPES)
@pytest.mark.parametrize("gate", ("none", "token", "sequence", "channel"))
@pytest.mark.parametrize("size", WIDTHS)
def test_norms_and_gradient(tfno, types, gate, size):
    activation = ("none", "silu", "sigmoid")[sum(size) % 3]
    check_between(tfno, between_inputs(*types, *size, gate, activation), f"[case] norms {types} {gate} {activation} {size}")


@pytest.mark.parametrize("types", TYPES)
@pytest.mark.parametrize("gate", ("none", "token", "sequence", "channel"))
@pytest.mark.parametrize("size", [(3, 2100, 64), (900, 5, 40), (2, 1300, 256), (5000, 1, 24), (40, 70, 1024)])
def test_norms_of_many_rows(tfno, types, gate, size):
    check_between(tfno, between_inputs(*types, *size, gate, "silu", seed=1), f"[case] rows {types} {gate} {size}")


@pytest.mark.parametrize("dtype", (F32, BF16))
@pytest.mark.parametrize("C", (48, 205, 4096))
@pytest.mark.parametrize("parts", ("no residual", "no norm after", "residual alone", "norm alone", "neither"))
def test_parts_of_the_norms(tfno, dtype, C, parts):
    x = between_inputs(dtype, None if parts == "no residual" else F32, 2, 19, C, "none" if parts in ("norm alone", "neither") else "token", "sigmoid", seed=2,
                       after=parts not in ("no norm after", "neither"))
    which = {"residual alone": (True, False), "norm alone": (False, True)}.get(parts, (True, True))
    if parts == "neither":
        x["w_before"] = None
    check_between(tfno, x, f"[case] parts {dtype} {C} {parts}", which)


@pytest.mark.parametrize("types", TYPES)
@pytest.mark.parametrize("gate", ("token", "sequence", "channel"))
@pytest.mark.parametrize("C", (40, 100, 1024))
def test_norms_lengths_and_what_stands_past_them(tfno, types, gate, C):
    B, T = 6, 50
    x = between_inputs(*types, B, T, C, gate, "silu", seed=3)
    x["ways"]["lengths"] = torch.tensor([T, 0, 1, 33, T + 9, -2], dtype=torch.int32, device="cuda")
    live = oracle.live_of(x["ways"]["lengths"], B, T, "cuda")[..., 0]
    for n in ("y", "r", "d_r", "d_n") + (("gate",) if gate == "token" else ()):
        x[n][~live] = float("nan")
    out, d = check_between(tfno, x, f"[case] norms lengths {types} {gate} {C}")
    for t in out + d[:2] + (d[2:3] if gate == "token" else []):
        assert (t[~live] == 0).all()
    if gate == "sequence":
        assert (d[2][1] == 0).all()


@pytest.mark.parametrize("dtype", (F32, BF16))
def test_norms_of_rows_of_zeros_and_of_nans(tfno, dtype):
    """A row of zeros stays one and has finite gradients; a NaN stays in its row, but for the sums over rows."""
    x = between_inputs(dtype, F32, 2, 12, 96, "token", "silu", seed=4)
    x["y"][:, 3] = 0
    x["r"][:, 3] = 0
    out, d = check_between(tfno, x, f"[case] zeros {dtype}")
    assert (out[0][:, 3] == 0).all() and (out[1][:, 3] == 0).all()
    x["y"][0, 5, 7] = float("nan")
    x["r"][1, 6, 2] = math.inf
    out2 = [torch.empty_like(t) for t in out]
    tfno.block_norm(*(x[n] for n in PARTS), *out2, **x["ways"])
    d2 = [torch.empty_like(t) for t in d]
    tfno.block_norm_backward(*(x[n] for n in PARTS), x["d_r"], x["d_n"], *d2, **x["ways"])
    keep = torch.ones(2, 12, dtype=torch.bool, device="cuda")
    keep[0, 5] = keep[1, 6] = False
    assert all(torch.equal(a[keep], b[keep]) for a, b in zip(out + d[:3], out2 + d2[:3]))
    assert torch.isnan(out2[1][0, 5]).all() and torch.isnan(d2[0][0, 5]).all()


@pytest.mark.parametrize("types", TYPES)
@pytest.mark.parametrize("C", (64, 100, 1024))
def test_norms_in_place_and_strides(tfno, types, C):
    dtype, res = types
    x = between_inputs(*types, 3, 21, C, "token", "silu", seed=5)
    w = between_wanted(x)
    y, r = x["y"].clone(), x["r"].clone()
    tfno.block_norm(y, r, *(x[n] for n in PARTS[2:]), r, y, **x["ways"])
    say(f"[case] in place {types} {C}")
    near("r", r, w[0], oracle.REL[res])
    near("n", y, w[1], oracle.REL[dtype])
    d_r, d_n, dgate = x["d_r"].clone(), x["d_n"].clone(), empty(x["gate"])
    tfno.block_norm_backward(*(x[n] for n in PARTS), d_r, d_n, d_n, d_r, dgate, None, None, **x["ways"])
    near("dy", d_n, w[2], oracle.REL_GATES[BF16] if dtype == BF16 else oracle.REL_SUMS)
    near("dr", d_r, w[3], oracle.REL_GATES[BF16] if res == BF16 else oracle.REL_SUMS)
    for more in (3, 8):
        z = dict(x)
        for n in ("y", "r", "gate", "d_r", "d_n"):
            wide = torch.full((21, 3, C + more), float("nan"), dtype=x[n].dtype, device="cuda").transpose(0, 1)[..., :C]
            z[n] = wide.copy_(x[n])
        out, d = check_between(tfno, z, f"[case] wide rows {more}")
    z = dict(x, gate=x["gate"][:, :1].expand(-1, 21, -1), r=x["r"][:1].expand(3, -1, -1))
    out = [empty(x["y"], res), empty(x["y"])]
    tfno.block_norm(*(z[n] for n in PARTS), *out, **x["ways"])
    w = between_wanted(z)
    near("repeated r", out[0], w[0], oracle.REL[res])
    near("repeated n", out[1], w[1], oracle.REL[dtype])


def test_norms_of_nothing(tfno):
    e = torch.empty(0, 4, 16, device="cuda")
    for gate, shape in ((torch.ones(16, device="cuda"), (16,)), (torch.ones(0, 16, device="cuda"), (0, 16))):
        dw, dgate = [torch.full((16,), 7.0, device="cuda") for _ in range(2)], torch.full(shape, 7.0, device="cuda")
        tfno.block_norm(e, e.clone(), gate, None, None, e.clone(), e.clone())
        tfno.block_norm_backward(e, e.clone(), gate, None, None, e.clone(), e.clone(), e.clone(), e.clone(), dgate, *dw)
        assert (dw[0] == 0).all() and (dw[1] == 0).all() and (dgate == 0).all()
    e, dgate = torch.empty(3, 0, 16, device="cuda"), torch.full((3, 16), 7.0, device="cuda")
    tfno.block_norm_backward(e, e.clone(), torch.ones(3, 16, device="cuda"), None, None, e.clone(), e.clone(), e.clone(), e.clone(), dgate, None, None)
    assert (dgate == 0).all()


def test_norms_gradient_against_differences(tfno):
    x = between_inputs(F32, F32, 2, 9, 40, "token", "silu", seed=6)
    d = [empty(x[n]) for n in PARTS]
    tfno.block_norm_backward(*(x[n] for n in PARTS), x["d_r"], x["d_n"], *d, **x["ways"])

    def loss(x):
        out = [empty(x["y"]), empty(x["y"])]
        tfno.block_norm(*(x[n] for n in PARTS), *out, **x["ways"])
        return float((out[0].double() * x["d_r"].double()).sum() + (out[1].double() * x["d_n"].double()).sum())

    for n, g in zip(PARTS, d):
        step = (g.double() / g.double().norm() * (0.02 * float(x[n].norm()))).float()
        slopes = [(loss(dict(x, **{n: x[n] + h * step})) - loss(dict(x, **{n: x[n] - h * step}))) / (2 * h) for h in (1.0, 0.5)]
        slope, want = (4 * slopes[1] - slopes[0]) / 3, float((g.double() * step.double()).sum())
        say(n, slope, want)
        assert abs(slope - want) <= 1e-2 * abs(want), n


def test_norms_equal_calls_give_equal_bits(tfno):
    for gate in ("token", "sequence", "channel"):
        x = between_inputs(BF16, F32, 4, 700, 136, gate, "silu", seed=7)
        runs = []
        for _ in range(2):
            d = [empty(x[n]) for n in PARTS]
            tfno.block_norm_backward(*(x[n] for n in PARTS), x["d_r"], x["d_n"], *d, **x["ways"])
            runs.append(d)
        assert all(torch.equal(a, b) for a, b in zip(*runs))


# ---------------------------------------------------------------- clipping

def wanted_clip(tensors, limit):
    total = math.sqrt(sum(float(torch.view_as_real(t).double().square().sum() if t.is_complex() else t.double().square().sum()) for t in tensors))
    scale = limit / total if total > limit else 1.0
    return total, [torch.view_as_real(t).double() * scale if t.is_complex() else t.double() * scale for t in tensors]


@pytest.mark.parametrize("limit", (0.0, 0.3, 1e9, math.inf))
@pytest.mark.parametrize("count", (1, 5, 130, 300))
def test_clip(tfno, count, limit):
    gen = torch.Generator("cuda").manual_seed(count)
    sizes = [(1,), (4097,), (3, 5, 7), (0,), (128, 257), (100000,), (16384,), (2, 8192)]
    tensors = []
    for i in range(count):
        t = torch.randn(*sizes[i % len(sizes)], generator=gen, device="cuda") * 10.0 ** -(i % 4)
        tensors.append(t.to(BF16) if i % 3 == 1 else torch.complex(t, -t) if i % 7 == 2 else t)
    if count > 1:
        tensors[0] = torch.randn(5000, generator=gen, device="cuda").to(BF16)[1:]          # not aligned to 16 bytes
        tensors[-1] = torch.randn(30, 20, generator=gen, device="cuda").t()                # axes in another order
    want, scaled = wanted_clip(tensors, limit)
    before = [t.clone() for t in tensors]
    norm = torch.empty((), device="cuda")
    tfno.clip_grad_norm(tensors, limit, norm)
    say(f"[case] clip {count} {limit} {want}")
    assert abs(float(norm) - want) <= 2.0 ** -23 * want
    for t, b, w in zip(tensors, before, scaled):
        if limit >= 1e9:
            assert torch.equal(t, b)
        elif t.numel():
            near(str(t.dtype), torch.view_as_real(t) if t.is_complex() else t, w, (2.0 ** -8 if t.dtype == BF16 else 2.0 ** -24) * (1 + 2.0 ** -10))


def test_clip_values_at_the_ends_of_their_range(tfno):
    for size in (1e30, 1e-30, 3e38, 1e-40):
        tensors = [torch.full((1000,), size, device="cuda"), torch.full((3,), -size, device="cuda")]
        want, scaled = wanted_clip(tensors, size)
        norm = torch.empty(1, device="cuda")
        tfno.clip_grad_norm(tensors, size, norm)
        if want < 3.4e38:
            assert abs(float(norm) - want) <= max(2.0 ** -23 * want, 2.0 ** -149)
        for t, w in zip(tensors, scaled):
            assert (t.double() - w).abs().max() <= max(2.0 ** -23 * float(w.abs().max()), 2.0 ** -149)


@pytest.mark.parametrize("bad", (math.nan, math.inf, -math.inf))
def test_clip_leaves_what_has_no_finite_norm(tfno, bad):
    tensors = [torch.randn(1000, device="cuda"), torch.randn(70, device="cuda").to(BF16)]
    tensors[1][3] = bad
    before, norm = [t.clone() for t in tensors], torch.empty((), device="cuda")
    tfno.clip_grad_norm(tensors, 0.5, norm)
    assert not math.isfinite(float(norm))
    assert all(torch.equal(t.nan_to_num(7.0), b.nan_to_num(7.0)) for t, b in zip(tensors, before))


def test_clip_of_nothing(tfno):
    norm = torch.empty((), device="cuda")
    tfno.clip_grad_norm([], 1.0, norm)
    assert float(norm) == 0
    tfno.clip_grad_norm([torch.empty(0, device="cuda")], 1.0, norm.fill_(3.0))
    assert float(norm) == 0
    assert tfno.clip_grad_norm([], 1.0) is None


def test_clip_does_not_touch_what_lies_beside(tfno):
    memory = torch.ones(40000, device="cuda")
    tfno.clip_grad_norm([memory[3:5000], memory[5001:5002], memory[20000:39999]], 1e-3)
    kept = torch.cat([memory[:3], memory[5000:5001], memory[5002:20000], memory[39999:]])
    assert (kept == 1).all() and (memory[3:5000] < 1).all() and float(memory[5001]) < 1


# ---------------------------------------------------------------- together

def block(tfno, p, u, r):
    """One block along time on u [B, T, C] with residual r, and all gradients of sum(r_out) + sum(n_out)."""
    B, T, C = u.shape
    x, gate, input_gate = (torch.matmul(u, w) for w in p["w"])
    y, r_out, n_out = (torch.empty_like(u) for _ in range(3))
    tape = tfno.gated_recurrence_tape(x)
    tfno.gated_recurrence(x, gate, input_gate, p["rate"], y, normalise=True, tape=tape)
    parts = (y, r, p["gate"], p["w_after"], p["w_before"])
    tfno.block_norm(*parts, r_out, n_out)
    ones = torch.ones_like(u)
    dy, dr = torch.empty_like(u), torch.empty_like(u)
    sums = [torch.empty_like(p[n]) for n in ("gate", "w_after", "w_before")]
    tfno.block_norm_backward(*parts, ones, ones, dy, dr, *sums)
    dx, dgate, dinput = (torch.empty_like(u) for _ in range(3))
    drate = torch.empty_like(p["rate"])
    tfno.gated_recurrence_backward(x, gate, input_gate, p["rate"], dy, dx, dgate, dinput, drate, tape, normalise=True)
    dw = [torch.matmul(u.reshape(-1, C).t().contiguous(), d.reshape(-1, C)) for d in (dx, dgate, dinput)]
    grads = [*dw, drate, *sums]
    norm = torch.empty((), device="cuda")
    tfno.clip_grad_norm(grads, 0.1, norm)
    return [r_out, n_out, dr, norm, *grads]


def parameters(C, gen):
    def normal(*shape):
        return torch.randn(*shape, generator=gen, device="cuda")
    return {"w": [normal(C, C) * C ** -0.5 for _ in range(3)], "rate": torch.exp(normal(C)), "gate": normal(C), "w_after": 1 + 0.1 * normal(C), "w_before": 1 + 0.1 * normal(C)}


def test_a_block_and_its_clipped_gradients(tfno):
    """The operators as a training step uses them, against autograd in float64."""
    gen = torch.Generator("cuda").manual_seed(5)
    B, T, C = 3, 140, 48
    p = parameters(C, gen)
    u, r = torch.randn(B, T, C, generator=gen, device="cuda"), torch.randn(B, T, C, generator=gen, device="cuda")
    got = block(tfno, p, u, r)
    leaves = [t.double().cpu().requires_grad_() for t in (*p["w"], p["rate"], p["gate"], p["w_after"], p["w_before"])]
    u, r = u.double().cpu(), r.double().cpu()
    x, gate, input_gate = (u @ w for w in leaves[:3])
    l = -leaves[3] * torch.sigmoid(gate)
    add = x * torch.sigmoid(input_gate) * torch.sqrt(-torch.expm1(2 * l))
    h, ys = torch.zeros(B, C, dtype=torch.float64), []
    for t in range(T):
        h = l[:, t].exp() * h + add[:, t]
        ys.append(h)
    y = torch.stack(ys, 1)
    r_out = r + leaves[4] * y / torch.sqrt((y * y).mean(-1, keepdim=True) + 1e-6) * leaves[5]
    n_out = r_out / torch.sqrt((r_out * r_out).mean(-1, keepdim=True) + 1e-6) * leaves[6]
    grads = torch.autograd.grad(r_out.sum() + n_out.sum(), leaves)
    norm = math.sqrt(sum(float(g.square().sum()) for g in grads))
    # the products in between are the library's, in float32: sums of 48 and 420 terms, so four times the bound of a sum
    near("r_out", got[0].cpu(), r_out.detach(), oracle.REL_SUMS)
    near("n_out", got[1].cpu(), n_out.detach(), oracle.REL_SUMS)
    assert abs(float(got[3]) - norm) <= oracle.REL_SUMS * 4 * norm
    for n, g, w in zip(("wx", "wgate", "winput", "rate", "gate", "w_after", "w_before"), got[4:], grads):
        near(n, g.cpu(), w * (0.1 / norm), 4 * oracle.REL_SUMS)


def test_another_stream_and_a_graph(tfno):
    """The run of operators on a stream of its own, and captured and replayed on new inputs between eager calls of the same workspace."""
    gen = torch.Generator("cuda").manual_seed(6)
    p = parameters(64, gen)
    data = [[torch.randn(2, 1300, 64, generator=gen, device="cuda") for _ in range(2)] for _ in range(4)]
    eager = [[t.clone() for t in block(tfno, p, *d)] for d in data]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = block(tfno, p, *data[0])
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, eager[0]))
    u, r = (t.clone() for t in data[0])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = block(tfno, p, u, r)
    for d, want in zip(data * 2, eager * 2):
        u.copy_(d[0]), r.copy_(d[1])
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want))
        assert all(torch.equal(a, b) for a, b in zip(block(tfno, p, *data[1]), eager[1]))


def test_two_graphs_share_the_workspace(tfno):
    """Two captured runs of different sizes, replayed by turns with eager calls between them: nothing is expected to be left of an earlier call."""
    gen = torch.Generator("cuda").manual_seed(7)
    runs = []
    for C, T in ((32, 1500), (80, 300)):
        p = parameters(C, gen)
        u, r = torch.randn(2, T, C, generator=gen, device="cuda"), torch.randn(2, T, C, generator=gen, device="cuda")
        want = [t.clone() for t in block(tfno, p, u, r)]
        runs.append((p, u, r, want))
    for p, u, r, _ in runs:                                     # the larger workspace is there before anything is captured
        block(tfno, p, u, r)
    torch.cuda.synchronize()
    graphs = []
    for p, u, r, _ in runs:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            graphs.append((graph, block(tfno, p, u, r)))
    for turn in range(6):
        graph, out = graphs[turn % 2]
        for t in out:
            t.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, runs[turn % 2][3])), turn
        p, u, r, want = runs[(turn + 1) % 2]
        assert all(torch.equal(a, b) for a, b in zip(block(tfno, p, u, r), want)), turn


def test_more_sequences_than_one_launch_takes(tfno):
    B = 2 ** 21 + 3
    gen = torch.Generator("cuda").manual_seed(8)
    x, gate = torch.randn(B, 2, 1, generator=gen, device="cuda"), -torch.rand(B, 2, 1, generator=gen, device="cuda")
    h, y, final = torch.randn(B, 1, generator=gen, device="cuda"), torch.empty(B, 2, 1, device="cuda"), torch.empty(B, 1, device="cuda")
    tape = tfno.gated_recurrence_tape(x)
    tfno.gated_recurrence(x, gate, None, None, y, initial_state=h, final_state=final, tape=tape)
    a = gate.double().exp()
    first = a[:, 0] * h.double() + x[:, 0].double()
    near("y", y, torch.stack((first, a[:, 1] * first + x[:, 1].double()), 1), oracle.REL[F32])
    assert torch.equal(final, y[:, 1])
    dx, dgate, d_initial = torch.empty_like(x), torch.empty_like(x), torch.empty_like(h)
    tfno.gated_recurrence_backward(x, gate, None, None, torch.ones_like(x), dx, dgate, None, None, tape, d_initial_state=d_initial)
    near("dx", dx, torch.stack((1 + a[:, 1], torch.ones_like(a[:, 1])), 1), oracle.REL[F32])
    near("dinitial", d_initial, a[:, 0] * (1 + a[:, 1]), oracle.REL[F32])
    states, o = h.clone(), torch.empty(B, 1, device="cuda")
    tfno.gated_recurrence_step(x[:, 0], gate[:, 0], None, None, states, o)
    assert torch.equal(states, o)
    near("step", o, first, oracle.REL[F32])


def test_norms_offsets_past_32_bits(tfno):
    far, T, C = 2 ** 31 + 64, 9, 64
    memory = torch.empty(far + 2 * T * C, dtype=BF16, device="cuda")
    x = between_inputs(BF16, F32, 2, T, C, "token", "silu", seed=8)
    x["y"] = memory.as_strided((2, T, C), (far, C, 1)).copy_(x["y"])
    n = memory[T * C:].as_strided((2, T, C), (far, C, 1))
    r = empty(x["r"])
    tfno.block_norm(*(x[k] for k in PARTS), r, n, **x["ways"])
    w = between_wanted(x)
    near("r", r, w[0], oracle.REL[F32])
    near("n", n, w[1], oracle.REL[BF16])


def test_norms_gradient_without_sums_needs_no_workspace(tfno):
    x = between_inputs(BF16, F32, 3, 50, 96, "token", "silu", seed=9)
    d = [empty(x[n]) for n in PARTS]
    tfno.block_norm_backward(*(x[n] for n in PARTS), x["d_r"], x["d_n"], *d, **x["ways"])
    kept = tfno._workspace
    try:
        tfno.set_workspace(None)
        again = [empty(x[n]) for n in PARTS[:3]]
        tfno.block_norm_backward(*(x[n] for n in PARTS), x["d_r"], x["d_n"], *again, None, None, **x["ways"])
        assert tfno._workspace is None
    finally:
        tfno.set_workspace(kept)
    assert all(torch.equal(a, b) for a, b in zip(again, d))
