"""The norm of heads with rotation and the gated delta rule on the GPU against float64."""
import pytest
import torch

import time_oracle as oracle

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16


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


def inputs(dtype, B, T, Hk, Hv, Dk, Dv, seed=0, state=True, decay=1.0, alike=0.5):
    gen = torch.Generator("cuda").manual_seed(1000 + seed)

    def normal(*shape):
        return torch.randn(*shape, generator=gen, device="cuda")

    def unit(x):
        return x / x.norm(dim=-1, keepdim=True)

    x = {"q": unit(normal(B, T, Hk, Dk)).to(dtype), "k": unit(normal(B, T, Hk, Dk) + alike * normal(1, 1, Hk, Dk)).to(dtype),
         "v": normal(B, T, Hv, Dv).to(dtype), "g": -decay * torch.rand(B, T, Hv, generator=gen, device="cuda") * 0.3,
         "beta": torch.sigmoid(normal(B, T, Hv)), "scale": Dk ** -0.5, "initial": normal(B, Hv, Dk, Dv) if state else None, "lengths": None}
    x["d_o"], x["d_final"] = normal(B, T, Hv, Dv).to(dtype), normal(B, Hv, Dk, Dv)
    return x


def names(x, *n):
    return [x[i] for i in n]


def forward(tfno, x, tape=None, o=None):
    v, k = x["v"], x["k"]
    o = torch.full(v.shape, 7.0, dtype=v.dtype, device="cuda") if o is None else o
    final = torch.full((v.shape[0], v.shape[2], k.shape[3], v.shape[3]), 7.0, device="cuda")
    tfno.gated_delta_rule(*names(x, "q", "k", "v", "g", "beta"), o, scale=x["scale"], initial_state=x["initial"], final_state=final, lengths=x["lengths"],
                          tape=tape)
    return o, final


def backward(tfno, x, tape, grads=None, initial=True):
    d = grads or {n: None if x[n] is None else torch.full(x[n].shape, 7.0, dtype=x[n].dtype, device="cuda") for n in ("q", "k", "v", "g", "beta")}
    d["initial"] = torch.full((x["v"].shape[0], x["v"].shape[2], x["k"].shape[3], x["v"].shape[3]), 7.0, device="cuda") if initial else None
    tfno.gated_delta_rule_backward(*names(x, "q", "k", "v", "g", "beta", "d_o"), *names(d, "q", "k", "v", "g", "beta"), tape, scale=x["scale"],
                                   initial_state=x["initial"], d_final_state=x["d_final"], d_initial_state=d["initial"], lengths=x["lengths"])
    return d


def want(x, grads):
    a = names(x, "q", "k", "v", "g", "beta", "scale", "initial", "lengths")
    return oracle.rule(*a, *names(x, "d_o", "d_final")) if grads else oracle.rule(*a)


def check_forward(tfno, x, what):
    say(what)
    o, final = forward(tfno, x)
    wo, wfinal = want(x, False)
    near("o", o, wo, oracle.REL[o.dtype])
    near("final", final, wfinal, oracle.REL[F32])
    return o, final


def check_both(tfno, x, what):
    say(what)
    tape = tfno.gated_delta_rule_tape(x["q"], x["v"])
    o, final = forward(tfno, x, tape)
    d = backward(tfno, x, tape)
    w = want(x, True)
    near("o", o, w[0], oracle.REL[o.dtype])
    near("final", final, w[1], oracle.REL[F32])
    for n, v in zip(("q", "k", "v", "g", "beta", "initial"), w[2:]):
        if d[n] is not None:
            near("d" + n, d[n], v, oracle.REL_GATES if n in ("g", "beta") else oracle.REL[d[n].dtype])
    return o, final, d


# one token, around the sizes of tiles and chunks, several chunks; head sizes from 1, odd, around the sizes of blocks; shared key heads
SIZES = [(1, 1, 1, 1, 64, 64), (2, 2, 1, 1, 1, 1), (3, 15, 2, 2, 16, 16), (2, 17, 1, 3, 7, 5), (2, 31, 2, 4, 32, 33), (2, 33, 1, 1, 33, 32),
         (1, 63, 2, 2, 64, 17), (2, 64, 1, 2, 65, 64), (2, 65, 3, 3, 100, 130), (1, 129, 1, 1, 128, 256), (2, 200, 2, 4, 128, 128), (1, 300, 1, 4, 48, 80),
         (5, 96, 2, 2, 31, 31)]


@pytest.mark.parametrize("dtype", (F32, BF16))
@pytest.mark.parametrize("size", SIZES)
def test_rule_and_gradient(tfno, dtype, size):
    check_both(tfno, inputs(dtype, *size), f"[case] rule {dtype} {size}")


@pytest.mark.parametrize("dtype", (F32, BF16))
@pytest.mark.parametrize("size", SIZES)
def test_rule_without_tape_gives_what_it_gives_with_one(tfno, dtype, size):
    x = inputs(dtype, *size, seed=1, state=False)
    o, final = check_forward(tfno, x, f"[case] no tape {dtype} {size}")
    o2, final2 = forward(tfno, x, tfno.gated_delta_rule_tape(x["q"], x["v"]))
    near("o with a tape", o2, o.double(), oracle.REL[dtype])
    near("final with a tape", final2, final.double(), oracle.REL[F32])


@pytest.mark.parametrize("dtype", (F32, BF16))
@pytest.mark.parametrize("size", [(1, 700, 1, 1, 64, 64), (40, 70, 8, 16, 128, 128), (64, 70, 8, 8, 64, 64), (9, 90, 32, 32, 32, 256), (2, 1500, 1, 2, 128, 64)])
def test_rule_of_many_heads_and_of_long_sequences(tfno, dtype, size):
    check_both(tfno, inputs(dtype, *size, seed=2), f"[case] large {dtype} {size}")


@pytest.mark.parametrize("dtype, size", [(BF16, (300, 520, 2, 4, 64, 64)), (F32, (101, 260, 4, 8, 40, 60))])
def test_batches_in_pieces(tfno, dtype, size):
    """So large a batch that it goes through the two kernels piece by piece: every sequence with its own lengths, first and last state."""
    x = inputs(dtype, *size, seed=13)
    B, T = size[:2]
    x["lengths"] = torch.randint(0, T + 1, (B,), generator=torch.Generator().manual_seed(5)).to(torch.int32).cuda()
    o, final = check_forward(tfno, x, f"[case] pieces {dtype} {size}")
    last = dict(x, lengths=x["lengths"][-3:].contiguous(), initial=x["initial"][-3:].contiguous())
    for n in ("q", "k", "v", "g", "beta"):
        last[n] = x[n][-3:]
    o2, final2 = forward(tfno, last)
    near("o of the last ones by themselves", o2, o[-3:].double(), oracle.REL[dtype])
    near("their states", final2, final[-3:].double(), oracle.REL[F32])


@pytest.mark.parametrize("dtype", (F32, BF16))
def test_gates_at_their_ends(tfno, dtype):
    x = inputs(dtype, 2, 150, 2, 2, 64, 48, seed=3)
    g, beta = x["g"], x["beta"]
    g[0, ::7] = float("-inf")                                  # forgets
    g[0, 3::11] = torch.finfo(F32).min
    g[1, :, 0] = 0.0                                           # never forgets
    g[1, ::5, 1] = -200.0
    beta[0, ::3] = 0.0                                         # writes nothing
    beta[1, ::4] = 1.0
    check_both(tfno, x, f"[case] gates {dtype}")
    x["g"][:] = float("-inf")
    check_both(tfno, x, f"[case] everything forgotten {dtype}")
    x["beta"][:] = 0.0
    check_both(tfno, x, f"[case] nothing written {dtype}")


@pytest.mark.parametrize("dtype", (F32, BF16))
@pytest.mark.parametrize("T, resets", [(128, (40,)), (200, (0, 3, 63, 64, 100, 101)), (700, (31, 32, 333, 640))])
def test_gradients_before_a_reset_do_not_see_what_follows(tfno, dtype, T, resets):
    """Sequences one after the other in one, each forgotten where the next begins, and the last one with 1e4 times the values and gradients: those of the ones before are as near as
    theirs alone.  The decay of a reset is 0, and so is its gradient."""
    x = inputs(dtype, 2, T, 1, 2, 64, 48, seed=24)
    for r in resets:
        x["g"][:, r] = float("-inf")
    for n in ("v", "d_o"):
        x[n][:, resets[-1]:] *= 1e4
    x["d_final"] *= 1e4
    say(f"[case] before a reset {dtype} {T} {resets}")
    tape = tfno.gated_delta_rule_tape(x["q"], x["v"])
    forward(tfno, x, tape)
    d = backward(tfno, x, tape)
    w = dict(zip(("o", "final", "q", "k", "v", "g", "beta", "initial"), want(x, True)))
    edges = [0, *resets, T]
    for first, last in zip(edges, edges[1:]):
        for n in ("q", "k", "v", "g", "beta"):
            if last > first:
                near(f"d{n} of {first} .. {last - 1}", d[n][:, first:last], w[n][:, first:last], oracle.REL_GATES if n in ("g", "beta") else oracle.REL[dtype])
    assert (d["g"][:, list(resets)] == 0).all()


@pytest.mark.parametrize("dtype", (F32, BF16))
def test_no_decay(tfno, dtype):
    x = inputs(dtype, 2, 130, 1, 2, 32, 32, seed=4)
    x["g"] = None
    check_both(tfno, x, f"[case] g None {dtype}")


@pytest.mark.parametrize("dtype", (F32, BF16))
def test_keys_that_are_all_alike(tfno, dtype):
    """The matrix of a chunk is then full below its diagonal: the inverse is well behaved, the powers of the matrix are not."""
    x = inputs(dtype, 1, 200, 2, 2, 64, 64, seed=5, decay=0.0)
    x["k"][:] = x["k"][:, :1]
    x["beta"][:] = 1.0
    check_both(tfno, x, f"[case] alike {dtype}")


@pytest.mark.parametrize("dtype", (F32, BF16))
@pytest.mark.parametrize("size", [(2, 64, 1, 2, 64, 64), (40, 64, 2, 2, 128, 128), (1, 640, 1, 1, 128, 64)])
def test_what_is_written_over_large_values(tfno, dtype, size):
    """One key of length one for every token and beta = 1: a token's value takes the place of the one before, and the outputs are the values.  The first state holds
    values a thousand times as large there, so what the outputs are made of (the products with the state and with the errors) cancels to a thousandth.  The bound: the rounding of
    the outputs, and of some ten sums in float32 (a matrix instruction adds 32 terms at once) with operands 2^-22 off at most, 16 * 2^-24 of the old values' size."""
    B, T, Hk, Hv, Dk, Dv = size
    x = inputs(dtype, *size, seed=14, decay=0.0)
    sign = torch.randn(1, 1, Hk, Dk, generator=torch.Generator("cuda").manual_seed(6), device="cuda").sign()
    key = 0.125 * sign * (torch.arange(Dk, device="cuda") < 64)          # 64 entries of 1 / 8
    for n in ("q", "k"):
        x[n][:] = key
    x["beta"][:] = 1.0
    old = 1000 * torch.randn(B, Hv, 1, Dv, generator=torch.Generator("cuda").manual_seed(7), device="cuda")
    x["initial"] = (key[0, 0].repeat_interleave(Hv // Hk, 0)[None, :, :, None] * old).contiguous()
    wo, wfinal = want(x, False)
    bound = 1000 * 16 * 2.0 ** -24
    for tape in (None, tfno.gated_delta_rule_tape(x["q"], x["v"])):
        say(f"[case] written over {dtype} {size} {tape is not None}")
        o, final = forward(tfno, x, tape)
        near("o", o[:, :64], wo[:, :64], (oracle.REL[BF16] if dtype is BF16 else 0) + bound)
        near("final", final, wfinal, bound)


@pytest.mark.parametrize("dtype", (F32, BF16))
@pytest.mark.parametrize("bad", (float("nan"), float("inf"), float("-inf")))
def test_lengths_and_what_stands_past_them(tfno, dtype, bad):
    B, T = 7, 140
    x = inputs(dtype, B, T, 2, 4, 48, 40, seed=6)
    x["lengths"] = torch.tensor([T, 0, 1, 64, 65, T + 50, -3], dtype=torch.int32, device="cuda")
    live = oracle.tokens_of(x["lengths"], B, T, "cuda")
    for n in ("q", "k", "v", "g", "beta", "d_o"):
        x[n][~live] = bad
    o, final, d = check_both(tfno, x, f"[case] lengths {dtype} {bad}")
    for t in (o, d["q"], d["k"], d["v"], d["g"], d["beta"]):
        assert (t[~live] == 0).all()
    assert torch.equal(final[1], x["initial"][1]) and torch.equal(final[6], x["initial"][6])
    assert torch.equal(d["initial"][1], x["d_final"][1])
    check_forward(tfno, x, "without tape")


@pytest.mark.parametrize("tokens", (1, 40))
def test_products_of_float32_are_not_off_to_one_side(tfno, tokens):
    """All factors 1 + 2^-7 - 2^-23, whose digits are ones where an operand's second and third part are: parts that are cut off lose 2^-21 of every product, all on one side.
    Nothing is written, so outputs are q times the state, and dq is d_o times it: one product of 32 terms, one rounding of at most 2^-23 and small ones below: 2^-22."""
    x = inputs(F32, 1, tokens, 1, 1, 32, 32, seed=18)
    for n in ("q", "initial", "d_o"):
        x[n][:] = 1 + 2.0 ** -7 - 2.0 ** -23
    x["beta"][:], x["g"], x["scale"] = 0.0, None, 1.0
    tape = tfno.gated_delta_rule_tape(x["q"], x["v"])
    want = 32 * (1 + 2.0 ** -7 - 2.0 ** -23) ** 2
    for o in (forward(tfno, x)[0], forward(tfno, x, tape)[0], backward(tfno, x, tape)["q"]):
        off = float((o.double() / want - 1).abs().max())
        say(f"   {off:.3g} of {2.0 ** -22:.3g}")
        assert off <= 2.0 ** -22


@pytest.mark.parametrize("dtype", (F32, BF16))
@pytest.mark.parametrize("T", (90, 128, 700))
@pytest.mark.parametrize("what", ("initial", "k", "v", "d_o", "d_final"))
def test_past_the_lengths_are_zeros_beside_a_nan(tfno, dtype, T, what):
    """A NaN in the state or in a token that counts: outputs and gradients of the tokens past the lengths are zeros all the same."""
    x = inputs(dtype, 3, T, 1, 2, 48, 40, seed=17)
    x["lengths"] = torch.tensor([70, 1, T - 1], dtype=torch.int32, device="cuda")
    x[what][:, 0] = float("nan")               # the first token, or the first head's state
    live = oracle.tokens_of(x["lengths"], 3, T, "cuda")
    tape = tfno.gated_delta_rule_tape(x["q"], x["v"])
    for o in (forward(tfno, x)[0], forward(tfno, x, tape)[0]):
        assert (o[~live] == 0).all()
        assert torch.isnan(o).any() == (what not in ("d_o", "d_final"))
    d = backward(tfno, x, tape)
    for n in ("q", "k", "v", "g", "beta"):
        assert (d[n][~live] == 0).all(), n
    assert torch.isnan(d["k"]).any()           # the one gradient that every input has a part in


@pytest.mark.parametrize("dtype", (F32, BF16))
@pytest.mark.parametrize("size", [(2, 150, 1, 2, 64, 48), (1, 70, 2, 8, 128, 128), (2, 200, 1, 3, 20, 33)])
def test_heads_that_share_keys_keep_their_gradients_apart(tfno, dtype, size):
    """The first value head of every key head has values and gradients 1e4 times the others', and then NaN: what the other heads get of their own is as near, and not NaN."""
    B, T, Hk, Hv, Dk, Dv = size
    group = Hv // Hk
    x = inputs(dtype, *size, seed=15)
    for n in ("v", "d_o"):
        x[n][:, :, ::group] *= 1e4
    for n in ("initial", "d_final"):
        x[n][:, ::group] *= 1e4
    say(f"[case] apart {dtype} {size}")
    tape = tfno.gated_delta_rule_tape(x["q"], x["v"])
    o, final = forward(tfno, x, tape)
    d = backward(tfno, x, tape)
    w = dict(zip(("o", "final", "q", "k", "v", "g", "beta", "initial"), want(x, True)))
    for n in ("q", "k"):
        near("d" + n, d[n], w[n], oracle.REL[dtype])
    for h in range(Hv):
        for n in ("v", "g", "beta"):
            near(f"d{n} of head {h}", d[n][:, :, h], w[n][:, :, h], oracle.REL_GATES if n != "v" else oracle.REL[dtype])
        near(f"o of head {h}", o[:, :, h], w["o"][:, :, h], oracle.REL[dtype])
    x["v"][:, 5, ::group] = float("nan")
    x["d_o"][:, T - 1, ::group] = float("nan")
    o2, final2 = forward(tfno, x, tape)
    d2 = backward(tfno, x, tape)
    rest = [h for h in range(Hv) if h % group]
    assert torch.isnan(o2[:, 5, 0]).all() and torch.isnan(d2["g"][:, 5, 0]).all()
    assert torch.equal(o2[:, :, rest], o[:, :, rest]) and torch.equal(final2[:, rest], final[:, rest])
    for n in ("v", "g", "beta"):
        assert torch.equal(d2[n][:, :, rest], d[n][:, :, rest]), n
    assert torch.equal(d2["initial"][:, rest], d["initial"][:, rest])


@pytest.mark.parametrize("dtype", (F32, BF16))
@pytest.mark.parametrize("size", [(1, 1100, 1, 1, 128, 128), (1, 1217, 2, 2, 64, 100), (3, 640, 1, 2, 33, 40), (2, 961, 1, 1, 100, 256), (4, 383, 1, 1, 16, 16)])
def test_few_heads_of_long_sequences(tfno, dtype, size):
    """So few heads that a sequence is cut into segments of chunks; ends inside a chunk, chunks that no segment is full of."""
    check_both(tfno, inputs(dtype, *size, seed=10), f"[case] segments {dtype} {size}")


@pytest.mark.parametrize("dtype", (F32, BF16))
@pytest.mark.parametrize("T", (700, 1089))
def test_lengths_of_few_heads(tfno, dtype, T):
    """Sequences that end in the first segment, in the middle, at a segment's edge and past all of them, with NaN behind their ends."""
    x = inputs(dtype, 7, T, 1, 2, 48, 40, seed=11)
    x["lengths"] = torch.tensor([T, 0, 1, T // 2, 256, T + 50, 513], dtype=torch.int32, device="cuda")
    live = oracle.tokens_of(x["lengths"], 7, T, "cuda")
    for n in ("q", "k", "v", "g", "beta", "d_o"):
        x[n][~live] = float("nan")
    o, final, d = check_both(tfno, x, f"[case] lengths of segments {dtype} {T}")
    for t in (o, d["q"], d["k"], d["v"], d["g"], d["beta"]):
        assert (t[~live] == 0).all()
    assert torch.equal(final[1], x["initial"][1]) and torch.equal(d["initial"][1], x["d_final"][1])
    check_forward(tfno, x, "without tape")


@pytest.mark.parametrize("dtype", (F32, BF16))
def test_segments_that_forget_all_or_nothing(tfno, dtype):
    x = inputs(dtype, 2, 900, 1, 1, 64, 64, seed=12)
    x["g"][0] = 0.0
    x["g"][1, ::100] = float("-inf")
    x["beta"][1, 300:700] = 0.0
    check_both(tfno, x, f"[case] segments at the gates' ends {dtype}")


def test_more_sequences_without_tokens_than_one_launch_takes(tfno):
    """2^25 walks of 192 threads: they go in pieces.  Every final state is the initial one."""
    x = inputs(F32, 2 ** 25, 0, 1, 1, 1, 1, seed=7)
    say("[case] 2^25 sequences of no tokens")
    assert torch.equal(forward(tfno, x)[1], x["initial"])


def test_no_tokens_at_all(tfno):
    x = inputs(F32, 3, 0, 2, 2, 16, 16, seed=7)
    tape = tfno.gated_delta_rule_tape(x["q"], x["v"])
    assert torch.equal(forward(tfno, x, tape)[1], x["initial"])
    assert torch.equal(backward(tfno, x, tape)["initial"], x["d_final"])
    x = inputs(F32, 0, 5, 2, 2, 16, 16, seed=7)
    forward(tfno, x)


@pytest.mark.parametrize("dtype", (F32, BF16))
@pytest.mark.parametrize("way", ("fused", "heads first", "one element off", "repeated", "wide rows"))
def test_strides(tfno, dtype, way):
    B, T, Hk, Hv, Dk, Dv = 2, 77, 2, 4, 64, 64
    x = inputs(dtype, B, T, Hk, Hv, Dk, Dv, seed=8)
    plain = dict(x)
    o, grads = None, None
    if way == "fused":          # slices of one projection, and gradients into slices of one tensor
        def fused():
            w = torch.empty(B, T, (2 * Hk + Hv) * Dk, dtype=dtype, device="cuda")
            q, k, v = w.split((Hk * Dk, Hk * Dk, Hv * Dv), -1)
            return q.unflatten(-1, (Hk, Dk)), k.unflatten(-1, (Hk, Dk)), v.unflatten(-1, (Hv, Dv))
        parts, dparts = fused(), fused()
        for n, p in zip("qkv", parts):
            p.copy_(x[n])
            x[n] = p
        gates = torch.empty(B, T, 2 * Hv, device="cuda")
        gates[..., :Hv], gates[..., Hv:] = x["g"], x["beta"]
        x["g"], x["beta"] = gates[..., :Hv], gates[..., Hv:]
        grads = {**dict(zip("qkv", dparts)), "g": torch.empty_like(plain["g"]), "beta": torch.empty_like(plain["g"])}
    elif way == "heads first":
        for n in ("q", "k", "v", "d_o", "g", "beta"):
            x[n] = x[n].transpose(1, 2).contiguous().transpose(1, 2)
        o = torch.empty(B, Hv, T, Dv, dtype=dtype, device="cuda").transpose(1, 2)
    elif way == "one element off":
        for n in ("q", "k", "v", "d_o", "g", "beta"):
            w = torch.empty(x[n].numel() + 1, dtype=x[n].dtype, device="cuda")[1:].view(x[n].shape)
            x[n] = w.copy_(x[n])
        o = torch.empty(plain["v"].numel() + 1, dtype=dtype, device="cuda")[1:].view(plain["v"].shape)
    elif way == "repeated":     # one trajectory's queries for the whole batch, one gate for all heads
        x["q"] = x["q"][:1].expand(B, -1, -1, -1)
        x["beta"] = x["beta"][..., :1].expand(-1, -1, Hv)
        x["d_o"] = x["d_o"][:, :1].expand(-1, T, -1, -1)
        grads = {n: torch.empty_like(plain[n]) for n in ("q", "k", "v", "g", "beta")}
    else:
        for n in ("q", "k", "v"):
            w = torch.empty(*x[n].shape[:-1], x[n].shape[-1] + 3, dtype=dtype, device="cuda")[..., :-3]
            x[n] = w.copy_(x[n])
    say(f"[case] strides {dtype} {way}")
    tape = tfno.gated_delta_rule_tape(x["q"], x["v"])
    got = forward(tfno, x, tape, o)
    d = backward(tfno, x, tape, grads)
    w = want(x, True)
    near("o", got[0], w[0], oracle.REL[dtype])
    near("final", got[1], w[1], oracle.REL[F32])
    for n, v in zip(("q", "k", "v", "g", "beta", "initial"), w[2:]):
        near("d" + n, d[n], v, oracle.REL_GATES if n in ("g", "beta") else oracle.REL[d[n].dtype])


@pytest.mark.parametrize("dtype", (F32, BF16))
def test_slices_that_interleave_by_heads(tfno, dtype):
    """Queries, keys and values of a head beside each other, normalised in place; results and gradients as the halves of rows."""
    B, T, H, D = 2, 77, 2, 64
    x = inputs(dtype, B, T, H, H, D, D, seed=16)
    packed = torch.stack([x[n] for n in "qkv"], 3)                        # [B, T, H, 3, D]
    gen = torch.Generator("cuda").manual_seed(8)
    cos, sin = torch.rand(T, D // 2, generator=gen, device="cuda"), torch.rand(T, D // 2, generator=gen, device="cuda")
    weight = torch.full((D,), D ** -0.5, device="cuda")                   # keys of length one
    normed = {n: oracle.norm(x[n], weight, cos, sin, None, 1e-6, False) for n in "qk"}
    x["q"], x["k"], x["v"] = packed.unbind(3)
    tfno.head_norm_rope(x["q"], x["k"], weight, weight, cos, sin, x["q"], x["k"])
    say(f"[case] by heads {dtype}")
    for n in "qk":
        near(n, x[n], normed[n], oracle.REL[dtype])
    rows = torch.empty(B, H, T, 2 * D, dtype=dtype, device="cuda").transpose(1, 2)
    rows[..., :D] = x["v"]
    x["v"], o = rows[..., :D], rows[..., D:]
    gates = torch.empty(B, T, H, 2, device="cuda")
    dqkv = torch.empty_like(packed)
    grads = {**dict(zip("qkv", dqkv.unbind(3))), "g": gates[..., 0], "beta": gates[..., 1]}
    tape = tfno.gated_delta_rule_tape(x["q"], x["v"])
    got = forward(tfno, x, tape, o)
    d = backward(tfno, x, tape, grads)
    w = want(x, True)
    near("o", got[0], w[0], oracle.REL[dtype])
    near("final", got[1], w[1], oracle.REL[F32])
    for n, v in zip(("q", "k", "v", "g", "beta", "initial"), w[2:]):
        near("d" + n, d[n], v, oracle.REL_GATES if n in ("g", "beta") else oracle.REL[d[n].dtype])


@pytest.mark.parametrize("dtype", (F32, BF16))
@pytest.mark.parametrize("way", ("fused", "heads first", "tokens first", "one element off", "repeated", "wide rows", "odd wide rows"))
@pytest.mark.parametrize("size", [(3, 77, 2, 4, 64, 64), (2, 130, 1, 2, 72, 40), (1, 700, 1, 1, 128, 96), (4, 65, 2, 2, 24, 32)])
def test_strides_without_a_tape(tfno, dtype, way, size):
    """Walks without a tape read BF16 keys and queries out of the caller's rows where these allow it, whole sequences and segments, to ends inside a chunk."""
    B, T, Hk, Hv, Dk, Dv = size
    x = inputs(dtype, *size, seed=19)
    if way == "fused":
        w = torch.empty(B, T, 2 * Hk * Dk + Hv * Dv, dtype=dtype, device="cuda")
        q, k, v = w.split((Hk * Dk, Hk * Dk, Hv * Dv), -1)
        for n, p in (("q", q.unflatten(-1, (Hk, Dk))), ("k", k.unflatten(-1, (Hk, Dk))), ("v", v.unflatten(-1, (Hv, Dv)))):
            x[n] = p.copy_(x[n])
    elif way in ("heads first", "tokens first"):
        axes = (1, 2) if way == "heads first" else (0, 1)
        for n in ("q", "k", "v", "g", "beta"):
            x[n] = x[n].transpose(*axes).contiguous().transpose(*axes)
    elif way == "one element off":
        for n in ("q", "k"):
            w = torch.empty(x[n].numel() + 1, dtype=dtype, device="cuda")[1:].view(x[n].shape)
            x[n] = w.copy_(x[n])
    elif way == "repeated":
        x["q"] = x["q"][:1].expand(B, -1, -1, -1)
        x["k"] = x["k"][:, :, :1].expand(-1, -1, Hk, -1)
    else:
        more = 8 if way == "wide rows" else 3
        for n in ("q", "k", "v"):
            w = torch.full((*x[n].shape[:-1], x[n].shape[-1] + more), float("nan"), dtype=dtype, device="cuda")[..., :-more]
            x[n] = w.copy_(x[n])
    check_forward(tfno, x, f"[case] strides without a tape {dtype} {way} {size}")
    x["lengths"] = torch.arange(T, T - 23 * B, -23, dtype=torch.int32, device="cuda")
    check_forward(tfno, x, "with lengths")


def test_offsets_past_32_bits(tfno):
    """Two trajectories further apart than 2^31 elements."""
    far, T, H, D = 2 ** 31 + 64, 70, 2, 64
    memory = torch.empty(far + 4 * T * H * D, dtype=BF16, device="cuda")
    x = inputs(BF16, 2, T, H, H, D, D, seed=9)
    views = [memory[i * T * H * D:].as_strided((2, T, H, D), (far, H * D, D, 1)) for i in range(4)]
    for n, w in zip(("q", "k", "v"), views):
        x[n] = w.copy_(x[n])
    say("[case] far apart")
    o, final = forward(tfno, x, o=views[3])
    wo, wfinal = want(x, False)
    near("o", o, wo, oracle.REL[BF16])
    near("final", final, wfinal, oracle.REL[F32])
    cos = torch.ones(T, D // 2, device="cuda")
    tfno.head_norm_rope(x["q"], x["k"], None, None, cos, torch.zeros_like(cos), views[3], views[2])
    near("norm", views[3], oracle.norm(x["q"], None, None, None, None, 1e-6, False), oracle.REL[BF16])


@pytest.mark.parametrize("dtype", (F32, BF16))
def test_gradient_against_differences(tfno, dtype):
    x = inputs(dtype, 2, 90, 1, 2, 24, 20, seed=10)
    tape = tfno.gated_delta_rule_tape(x["q"], x["v"])
    forward(tfno, x, tape)
    d = backward(tfno, x, tape)
    gen = torch.Generator("cuda").manual_seed(5)
    for n in ("q", "k", "v", "g", "beta", "initial"):
        way = torch.randn(x[n].shape, generator=gen, device="cuda", dtype=torch.float64)

        def loss(h):
            o, final = want({**x, n: x[n].double() + h * way}, False)
            return float((o * x["d_o"].double()).sum() + (final * x["d_final"].double()).sum())

        slope = (loss(1e-4) - loss(-1e-4)) / 2e-4
        got = float((d[n].double() * way).sum())
        # the error of a sum with a random direction is about the L2 error of the gradient: four standard deviations, and 1e-6 for the differences
        bound = 4 * oracle.REL_GATES if d[n].dtype == F32 else 4 * oracle.REL[BF16]
        say(f"   d{n}: {got:.8g}, by differences {slope:.8g}")
        assert abs(got - slope) <= bound * float(d[n].double().norm()) + 1e-6 * abs(slope)


@pytest.mark.parametrize("dtype", (F32, BF16))
def test_equal_calls_give_equal_bits_and_the_past_does_not_see_the_future(tfno, dtype):
    x = inputs(dtype, 3, 180, 2, 4, 64, 64, seed=11)
    tape = tfno.gated_delta_rule_tape(x["q"], x["v"])
    first, again = forward(tfno, x, tape), forward(tfno, x, tape)
    d, d2 = backward(tfno, x, tape), backward(tfno, x, tape)
    assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])
    assert all(torch.equal(d[n], d2[n]) for n in d)
    for n in ("q", "k", "v", "g", "beta"):
        x[n][:, 100:] = x[n][:, 100:] * 0.5
    assert torch.equal(first[0][:, :100], forward(tfno, x)[0][:, :100])


def test_another_stream_and_a_graph(tfno):
    x = inputs(BF16, 2, 100, 2, 2, 64, 64, seed=12)
    cos = torch.rand(100, 32, device="cuda")
    w = torch.rand(64, device="cuda")
    tape = tfno.gated_delta_rule_tape(x["q"], x["v"])
    qn, kn, o, final = torch.empty_like(x["q"]), torch.empty_like(x["k"]), torch.empty_like(x["v"]), torch.empty_like(x["initial"])
    d = {n: torch.empty_like(x[n]) for n in ("q", "k", "v", "g", "beta", "initial")}
    dw = torch.empty(2, 64, device="cuda")
    states, so = x["initial"].clone(), torch.empty_like(x["v"][:, 0])

    def work():
        tfno.head_norm_rope(x["q"], x["k"], w, w, cos, cos, qn, kn)
        tfno.gated_delta_rule(qn, kn, x["v"], x["g"], x["beta"], o, scale=0.1, initial_state=x["initial"], final_state=final, tape=tape)
        tfno.gated_delta_rule_backward(qn, kn, x["v"], x["g"], x["beta"], x["d_o"], d["q"], d["k"], d["v"], d["g"], d["beta"], tape, scale=0.1,
                                       initial_state=x["initial"], d_final_state=x["d_final"], d_initial_state=d["initial"])
        tfno.head_norm_rope_backward(x["q"], x["k"], w, w, cos, cos, d["q"], d["k"], d["q"], d["k"], dw[0], dw[1])
        states.copy_(x["initial"])
        tfno.gated_delta_rule_step(qn[:, 0], kn[:, 0], x["v"][:, 0], x["g"][:, 0], x["beta"][:, 0], states, so, scale=0.1)

    results = [qn, kn, o, final, dw, states, so, *d.values()]
    work()
    torch.cuda.synchronize()
    eager = [r.clone() for r in results]
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        for r in results:
            r.fill_(7.0)
        work()
    stream.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(eager, results))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        work()
    for step in range(4):
        for n in ("q", "v", "d_o"):
            x[n].mul_(-1.0)
        for r in results:
            r.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        replayed = [r.clone() for r in results]
        work()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(replayed, results)), step


# ---------------------------------------------------------------- one token

@pytest.mark.parametrize("dtype", (F32, BF16))
@pytest.mark.parametrize("size", [(1, 1, 1, 1, 1), (1, 4, 8, 64, 64), (3, 2, 2, 7, 5), (5, 1, 3, 33, 20), (2, 2, 4, 128, 256), (70, 4, 8, 100, 48), (2, 1, 1, 128, 130),
                                  (200, 4, 4, 128, 128), (1, 1, 2, 16, 3)])
def test_step(tfno, dtype, size):
    B, Hk, Hv, Dk, Dv = size
    x = inputs(dtype, B, 1, Hk, Hv, Dk, Dv, seed=20)
    pool = B + 3
    states = torch.randn(pool, Hv, Dk, Dv, generator=torch.Generator("cuda").manual_seed(1), device="cuda")
    slots = torch.randperm(pool, generator=torch.Generator("cuda").manual_seed(2), device="cuda")[:B].to(torch.int32)
    if B > 2:
        slots[1], slots[2] = -1, pool
        x["g"][0], x["beta"][0] = float("-inf"), 1.0
    before = states.clone()
    o = torch.full((B, Hv, Dv), 7.0, dtype=dtype, device="cuda")
    say(f"[case] step {dtype} {size}")
    tfno.gated_delta_rule_step(*(x[n][:, 0] for n in ("q", "k", "v", "g", "beta")), states, o, slots=slots, scale=x["scale"])
    live = [b for b in range(B) if 0 <= int(slots[b]) < pool]
    rows = slots[live].long()
    wo, wS = oracle.rule(*(x[n][live] for n in ("q", "k", "v", "g", "beta")), x["scale"], before[rows])
    near("o", o[live], wo[:, 0], oracle.REL[dtype])
    near("states", states[rows], wS, oracle.REL[F32])
    rest = [s for s in range(pool) if s not in set(rows.tolist())]
    assert torch.equal(states[rest], before[rest])
    if B > 2:
        assert (o[1] == 0).all() and torch.isnan(o[2]).all()


@pytest.mark.parametrize("dtype", (F32, BF16))
@pytest.mark.parametrize("size", [(3, 2, 4, 64, 64), (2, 1, 1, 100, 33), (600, 1, 2, 32, 48)])
def test_step_forgets_whatever_the_state_was(tfno, dtype, size):
    """g = -inf in a place of the pool that holds NaN and infinities: the state is the token's alone.  Other heads keep theirs."""
    B, Hk, Hv, Dk, Dv = size
    x = inputs(dtype, B, 1, Hk, Hv, Dk, Dv, seed=22)
    states = x["initial"].clone()
    x["g"][0] = float("-inf")
    states[0] = torch.tensor([float("nan"), float("inf"), float("-inf"), 1e38], device="cuda").repeat(states[0].numel() // 4 + 1)[:states[0].numel()].view(states[0].shape)
    x["initial"][0] = 0.0
    o = torch.full((B, Hv, Dv), 7.0, dtype=dtype, device="cuda")
    say(f"[case] forgets {dtype} {size}")
    tfno.gated_delta_rule_step(*(x[n][:, 0] for n in ("q", "k", "v", "g", "beta")), states, o, scale=x["scale"])
    wo, wS = want(x, False)
    near("o", o, wo[:, 0], oracle.REL[dtype])
    near("states", states, wS, oracle.REL[F32])


@pytest.mark.parametrize("dtype", (F32, BF16))
def test_steps_follow_the_whole_sequence(tfno, dtype):
    x = inputs(dtype, 2, 70, 2, 4, 64, 40, seed=21)
    states, outputs = x["initial"].clone(), []
    for t in range(70):
        o = torch.empty(2, 4, 40, dtype=dtype, device="cuda")
        tfno.gated_delta_rule_step(*(x[n][:, t] for n in ("q", "k", "v", "g", "beta")), states, o, scale=x["scale"])
        outputs.append(o)
    wo, wS = want(x, False)
    near("o", torch.stack(outputs, 1), wo, oracle.REL[dtype])
    near("state", states, wS, oracle.REL[F32])
    o = torch.empty(2, 4, 40, dtype=dtype, device="cuda")
    tfno.gated_delta_rule_step(x["q"][:, 0], x["k"][:, 0], x["v"][:, 0], None, x["beta"][:, 0], states, o)       # no decay, the default scale
    again = oracle.rule(x["q"][:, :1], x["k"][:, :1], x["v"][:, :1], None, x["beta"][:, :1], 64 ** -0.5, wS)
    near("o without decay", o, again[0][:, 0], oracle.REL[dtype])


@pytest.mark.parametrize("B, Hv", [(1, 2 ** 24 + 3), (2 ** 24 + 3, 1), (3, 2 ** 23 - 5)])
def test_step_of_more_heads_than_one_launch_takes(tfno, B, Hv):
    """2^24 workgroups of 256 threads are 2^32: such calls go in several launches."""
    gen = torch.Generator("cuda").manual_seed(23)
    q, k = (torch.randn(B, 1, 1, generator=gen, device="cuda") for _ in range(2))
    v, states = torch.randn(B, Hv, 1, generator=gen, device="cuda"), torch.randn(B, Hv, 1, 1, generator=gen, device="cuda")
    g, beta = -torch.rand(B, Hv, generator=gen, device="cuda"), torch.rand(B, Hv, generator=gen, device="cuda")
    o = torch.full_like(v, 7.0)
    Sb = states[..., 0].double() * g.double().exp()[..., None]
    S = Sb + (beta[..., None].double() * k.double()) * (v.double() - Sb * k.double())
    say(f"[case] step of {B} x {Hv} heads")
    tfno.gated_delta_rule_step(q, k, v, g, beta, states, o, scale=0.5)
    near("o", o, 0.5 * S * q.double(), oracle.REL[F32])
    near("states", states[..., 0], S, oracle.REL[F32])


# ---------------------------------------------------------------- norm with rotation

NORMS = [(1, 1, 1, 1, 1, 0), (2, 3, 2, 1, 2, 2), (1, 5, 3, 2, 3, 2), (2, 7, 4, 2, 7, 4), (1, 1, 8, 8, 64, 64), (3, 37, 6, 2, 80, 40), (2, 33, 2, 2, 96, 96),
         (2, 100, 16, 4, 128, 128), (1, 9, 5, 1, 128, 30), (2, 9, 1, 3, 200, 8), (1, 17, 2, 2, 256, 256), (1, 3, 1, 1, 511, 510), (2, 4, 2, 2, 512, 64),
         (4, 5, 0, 3, 64, 32), (4, 5, 3, 0, 64, 64)]


@pytest.mark.parametrize("dtype", (F32, BF16))
@pytest.mark.parametrize("interleaved", (False, True))
@pytest.mark.parametrize("size", NORMS)
def test_norm(tfno, dtype, interleaved, size):
    B, T, Hq, Hk, D, R = size
    gen = torch.Generator("cuda").manual_seed(30)

    def normal(*shape):
        return torch.randn(*shape, generator=gen, device="cuda")

    qk = (normal(B, T, Hq + Hk, D) * 3).to(dtype)
    dqk = normal(B, T, Hq + Hk, D).to(dtype)
    q, k, dy, dz = qk[:, :, :Hq], qk[:, :, Hq:], dqk[:, :, :Hq], dqk[:, :, Hq:]
    if T > 2 and Hq:
        q[:, 1, 0] = 0.0                              # a row of zeros has a norm too
    wq, wk = 1 + 0.3 * normal(D), 1 + 0.3 * normal(D)
    P = 3 * T
    angle = 6.3 * torch.rand(P, R // 2, generator=gen, device="cuda")
    cos, sin = (torch.cos(angle), torch.sin(angle)) if R else (None, None)
    for positions in (None, torch.randint(0, P, (B, T), generator=gen, device="cuda", dtype=torch.int32)):
        say(f"[case] norm {dtype} {interleaved} {size} {positions is not None}")
        yq, yk = torch.full_like(q, 7.0), torch.full_like(k, 7.0)
        tfno.head_norm_rope(q, k, wq, wk, cos, sin, yq, yk, positions=positions, eps=1e-4, interleaved=interleaved)
        dq, dk, dwq, dwk = torch.full_like(q, 7.0), torch.full_like(k, 7.0), torch.full_like(wq, 7.0), torch.full_like(wk, 7.0)
        tfno.head_norm_rope_backward(q, k, wq, wk, cos, sin, dy, dz, dq, dk, dwq, dwk, positions=positions, eps=1e-4, interleaved=interleaved)
        for n, x, w, d, got, dx, dw in (("q", q, wq, dy, yq, dq, dwq), ("k", k, wk, dz, yk, dk, dwk)):
            a = oracle.norm(x, w, cos, sin, positions, 1e-4, interleaved, d)
            near(n, got, a[0], oracle.REL[dtype])
            # one value a head: its gradient is the small difference of two that cancel
            near("d" + n, dx.double() + (x.double() if D == 1 else 0), a[1] + (x.double() if D == 1 else 0), oracle.REL[dtype])
            near("dw" + n, dw, a[2], oracle.REL[F32])


@pytest.mark.parametrize("dtype", (F32, BF16))
@pytest.mark.parametrize("interleaved", (False, True))
@pytest.mark.parametrize("size", [(8, 512, 13, 4, 128, 128), (8, 2049, 17, 3, 64, 32), (16, 260, 3, 7, 63, 20), (2, 4100, 1, 6, 100, 50), (700, 3, 5, 11, 200, 64), (1, 9000, 9, 0, 128, 64),
                                  (5, 5000, 0, 7, 48, 48)])
def test_norm_of_many_heads(tfno, dtype, interleaved, size):
    """So many heads that a group of lanes takes four of them, heads that are no multiple of four, more groups than the gradient's workgroups take in one turn; and heads too wide for that."""
    B, T, Hq, Hk, D, R = size
    gen = torch.Generator("cuda").manual_seed(36)

    def normal(*shape):
        return torch.randn(*shape, generator=gen, device="cuda")

    q, dy = (normal(B, T, Hq, D) * 3).to(dtype), normal(B, T, Hq, D).to(dtype)
    k, dz = (normal(B, T, Hk, D) * 3).to(dtype), normal(B, T, Hk, D).to(dtype)
    wq, wk = 1 + 0.3 * normal(D), 1 + 0.3 * normal(D)
    angle = 6.3 * torch.rand(2 * T, R // 2, generator=gen, device="cuda")
    cos, sin = torch.cos(angle), torch.sin(angle)
    positions = torch.randint(0, 2 * T, (B, T), generator=gen, device="cuda", dtype=torch.int32)
    say(f"[case] norm of many heads {dtype} {interleaved} {size}")
    yq, yk = torch.full_like(q, 7.0), torch.full_like(k, 7.0)
    tfno.head_norm_rope(q, k, wq, wk, cos, sin, yq, yk, positions=positions, interleaved=interleaved)
    dq, dk, dwq, dwk = torch.full_like(q, 7.0), torch.full_like(k, 7.0), torch.full_like(wq, 7.0), torch.full_like(wk, 7.0)
    tfno.head_norm_rope_backward(q, k, wq, wk, cos, sin, dy, dz, dq, dk, dwq, dwk, positions=positions, interleaved=interleaved)
    for n, x, w, d, got, dx, dw in (("q", q, wq, dy, yq, dq, dwq), ("k", k, wk, dz, yk, dk, dwk)):
        a = oracle.norm(x, w, cos, sin, positions, 1e-6, interleaved, d)
        near(n, got, a[0], oracle.REL[dtype])
        near("d" + n, dx, a[1], oracle.REL[dtype])
        near("dw" + n, dw, a[2], oracle.REL[F32])


def test_norm_in_place_without_weights_and_with_strides(tfno):
    gen = torch.Generator("cuda").manual_seed(31)
    cos, sin = torch.rand(9, 16, generator=gen, device="cuda"), torch.rand(9, 16, generator=gen, device="cuda")
    for dtype in (F32, BF16):
        w = torch.randn(2, 9, 4 * 32 + 5, generator=gen, device="cuda").to(dtype)
        for off in (0, 1, 4):                          # slices of wide rows, at odd places too
            q, k = w[..., off:off + 64].unflatten(-1, (2, 32)), w[..., off + 64:off + 128].unflatten(-1, (2, 32))
            wants = [oracle.norm(x, None, cos, sin, None, 1e-6, False) for x in (q, k)]
            dx = [oracle.norm(x, None, cos, sin, None, 1e-6, False, x)[1] for x in (q, k)]
            dq, dk = q.clone(), k.clone()              # gradients over the gradients that they come from
            tfno.head_norm_rope_backward(q, k, None, None, cos, sin, dq, dk, dq, dk)
            near("dq", dq, dx[0], oracle.REL[dtype])
            near("dk", dk, dx[1], oracle.REL[dtype])
            tfno.head_norm_rope(q, k, None, None, cos, sin, q, k)
            near("q", q, wants[0], oracle.REL[dtype])
            near("k", k, wants[1], oracle.REL[dtype])


def test_norm_of_positions_that_the_tables_do_not_hold(tfno):
    q = torch.randn(1, 4, 2, 12, device="cuda")
    out, k_out = torch.zeros_like(q), torch.zeros_like(q)
    cos = torch.ones(5, 4, device="cuda")
    positions = torch.tensor([[0, 5, -1, 4]], dtype=torch.int32, device="cuda")
    tfno.head_norm_rope(q, q, None, None, cos, torch.zeros_like(cos), out, k_out, positions=positions)
    assert torch.isnan(out[:, 1:3, :, :8]).all() and torch.isfinite(out[:, 1:3, :, 8:]).all()
    assert torch.isfinite(out[:, (0, 3)]).all()


def test_norm_gradient_against_differences(tfno):
    gen = torch.Generator("cuda").manual_seed(33)
    q, dy = torch.randn(2, 5, 3, 24, generator=gen, device="cuda"), torch.randn(2, 5, 3, 24, generator=gen, device="cuda")
    w = 1 + 0.2 * torch.randn(24, generator=gen, device="cuda")
    angle = torch.rand(5, 6, generator=gen, device="cuda")
    cos, sin = torch.cos(angle), torch.sin(angle)
    d = {"x": torch.empty_like(q), "w": torch.empty_like(w)}
    tfno.head_norm_rope_backward(q, q, w, w, cos, sin, dy, dy, d["x"], torch.empty_like(q), d["w"], None)
    for n in ("x", "w"):
        way = torch.randn(d[n].shape, generator=gen, device="cuda", dtype=torch.float64)

        def loss(h):
            return float((oracle.norm(q.double() + (h * way if n == "x" else 0), w.double() + (h * way if n == "w" else 0), cos, sin, None, 1e-6, False) * dy).sum())

        slope = (loss(1e-4) - loss(-1e-4)) / 2e-4
        assert abs(float((d[n].double() * way).sum()) - slope) <= 4 * oracle.REL_GATES * float(d[n].norm()) + 1e-6 * abs(slope)


@pytest.mark.parametrize("dtype", (F32, BF16))
@pytest.mark.parametrize("size", [(2, 9, 3, 1, 64, 32), (3, 200, 8, 2, 80, 40)])
def test_norm_gradient_without_the_weights_needs_no_workspace(tfno, dtype, size):
    B, T, Hq, Hk, D, R = size
    gen = torch.Generator("cuda").manual_seed(35)
    q, dy = (torch.randn(B, T, Hq, D, generator=gen, device="cuda").to(dtype) for _ in range(2))
    k, dz = (torch.randn(B, T, Hk, D, generator=gen, device="cuda").to(dtype) for _ in range(2))
    angle = torch.rand(T, R // 2, generator=gen, device="cuda")
    cos, sin = torch.cos(angle), torch.sin(angle)
    before = tfno._workspace
    try:
        tfno.set_workspace(None)
        dq, dk = torch.full_like(q, 7.0), torch.full_like(k, 7.0)
        tfno.head_norm_rope_backward(q, k, None, None, cos, sin, dy, dz, dq, dk)
        assert tfno._workspace is None
    finally:
        tfno.set_workspace(before)
    near("dq", dq, oracle.norm(q, None, cos, sin, None, 1e-6, False, dy)[1], oracle.REL[dtype])
    near("dk", dk, oracle.norm(k, None, cos, sin, None, 1e-6, False, dz)[1], oracle.REL[dtype])
    dw = torch.empty(D, device="cuda")
    for weights in ((dw, None), (None, dw)):
        tfno.head_norm_rope_backward(q, k, None, None, cos, sin, dy, dz, dq, dk, *weights)
        x, d = (q, dy) if weights[0] is dw else (k, dz)
        near("dw", dw, oracle.norm(x, None, cos, sin, None, 1e-6, False, d)[2], oracle.REL[F32])


def test_norm_of_nothing(tfno):
    q = torch.zeros(0, 4, 2, 16, device="cuda")
    dw = torch.full((16,), 7.0, device="cuda")
    tfno.head_norm_rope(q, q, None, None, None, None, q.clone(), q.clone())
    tfno.head_norm_rope_backward(q, q, None, None, None, None, q.clone(), q.clone(), q.clone(), q.clone(), dw, None)
    assert (dw == 0).all()


def test_norm_of_more_heads_than_one_launch_takes(tfno):
    """2^26 heads and a few, four a workgroup: 2^24 workgroups of 256 threads would be 2^32."""
    B, H, D = 2 ** 20 + 1, 64, 129
    gen = torch.Generator("cuda").manual_seed(34)
    x = torch.randn(1, 1, H, D, generator=gen, device="cuda").to(BF16)
    none = torch.empty(B, 1, 0, D, dtype=BF16, device="cuda")
    out = torch.full((B, 1, H, D), 7.0, dtype=BF16, device="cuda")
    say("[case] norm of 2^26 heads")
    tfno.head_norm_rope(x.expand(B, 1, H, D), none, None, None, None, None, out, none)
    near("the first", out[:1], oracle.norm(x, None, None, None, None, 1e-6, False), oracle.REL[BF16])
    assert all(torch.equal(part, out[:1].expand_as(part)) for part in out.split(1 << 17))
