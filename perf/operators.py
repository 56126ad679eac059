"""The operators that mix a trajectory of fields along time: the gated delta rule over whole sequences, its gradient and its step for
one token, and the norm of queries and keys for each head with the position rotation in the same pass.

``listed`` and ``draw`` give cases, ``prepare`` their inputs on the GPU, ``run`` one pass: with ``own`` false in elementary torch
operations in 32 bits, with ``own`` true through the framework's entry points.  ``exact`` gives the same in 64 bits from the
definition, token by token; ``work`` what a pass cannot do without.
"""
import math

import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
EPS = 1e-6


def listed():
    return [
        # one frame of a rollout: its queries and keys, one token of one trajectory
        _norm("norm one token", "norm", "bf16", B=1, T=1, Hq=8, Hk=8, D=64, R=64),
        # a head size and a rotated part that are no powers of two, float32 fields, grouped heads, neighbours paired, positions of its own
        _norm("norm odd f32", "norm", "f32", B=7, T=333, Hq=6, Hk=2, D=80, R=40, pairs="neighbours", positions=True),
        # a training batch: both directions, heads of 128
        _norm("norm train bf16", "norm_train", "bf16", B=16, T=1024, Hq=16, Hk=8, D=128, R=128),
        # one step of a single trajectory, where latency counts
        _rule("step one", "step", "bf16", B=1, T=1, Hk=4, Hv=8, Dk=64, Dv=64),
        # a serving step of many trajectories out of a larger pool of states
        _rule("step many", "step", "bf16", B=256, T=1, Hk=16, Hv=16, Dk=128, Dv=128),
        # pencils of 1024 points of a batch of 256 with 128 channels, read as sequences of two heads
        _rule("rule batch bf16", "rule", "bf16", B=256, T=1024, Hk=2, Hv=2, Dk=64, Dv=64),
        # one long trajectory with few heads, from a state that an earlier part left
        _rule("rule long bf16", "rule", "bf16", B=1, T=16384, Hk=4, Hv=8, Dk=128, Dv=128, state=True),
        # float32 fields of odd sizes, trajectories of different lengths
        _rule("rule odd f32", "rule", "f32", B=5, T=777, Hk=3, Hv=3, Dk=48, Dv=80, ragged=True, state=True),
        # a short context with float32 fields
        _rule("rule short f32", "rule", "f32", B=32, T=100, Hk=8, Hv=8, Dk=64, Dv=64, state=True),
        # training: value heads that share key heads
        _rule("train bf16", "rule_train", "bf16", B=4, T=2048, Hk=8, Hv=16, Dk=128, Dv=128),
        # training on float32 fields, trajectories of different lengths, a learned first state
        _rule("train ragged f32", "rule_train", "f32", B=16, T=300, Hk=8, Hv=8, Dk=64, Dv=64, ragged=True, state=True),
        # the smallest training step: few short trajectories
        _rule("train small bf16", "rule_train", "bf16", B=2, T=129, Hk=4, Hv=4, Dk=64, Dv=64, state=True),
    ]


def _norm(name, op, dtype, B, T, Hq, Hk, D, R, pairs="halves", positions=False):
    c = {"op": op, "dtype": dtype, "B": B, "T": T, "Hq": Hq, "Hk": Hk, "D": D, "R": R, "pairs": pairs, "positions": positions}
    return {"name": name, **c} if name else c


def _rule(name, op, dtype, B, T, Hk, Hv, Dk, Dv, ragged=False, state=False):
    c = {"op": op, "dtype": dtype, "B": B, "T": T, "Hk": Hk, "Hv": Hv, "Dk": Dk, "Dv": Dv, "ragged": ragged, "state": state}
    return {"name": name, **c} if name else c


def _log(rng, low, high):
    return max(low, min(high, round(math.exp(rng.uniform(math.log(low), math.log(high))))))


def _cost(case):
    w = work(case)
    return max(w["bytes"], w["flops"] / 50)


def draw(rng):
    op = rng.choice(("norm", "norm_train", "step", "rule", "rule", "rule_train", "rule_train"))
    dtype = rng.choice(("f32", "bf16"))
    most = max(_cost(c) for c in listed() if c["op"] == op)
    if op in ("norm", "norm_train"):
        most = max(_cost(c) for c in listed() if c["op"] == "norm_train")
        D = rng.choice((rng.randint(16, 128), 32, 64, 128, 256))
        c = _norm("", op, dtype, B=_log(rng, 1, 64), T=_log(rng, 1, 2048), Hq=_log(rng, 1, 32), Hk=_log(rng, 1, 8), D=D,
                  R=rng.choice((D // 2 * 2, 2 * rng.randint(1, D // 2))), pairs=rng.choice(("halves", "neighbours")), positions=rng.random() < 0.5)
    else:
        Hk, Dk, Dv = _log(rng, 1, 16), rng.choice((rng.randint(16, 128), 32, 64, 128)), rng.choice((rng.randint(16, 128), 64, 128))
        T = 1 if op == "step" else _log(rng, 1, 16384 if op == "rule" else 4096)
        c = _rule("", op, dtype, B=_log(rng, 1, 256), T=T, Hk=Hk, Hv=Hk * rng.choice((1, 1, 2, 4)), Dk=Dk, Dv=Dv,
                  ragged=op != "step" and rng.random() < 0.5, state=op != "step" and rng.random() < 0.5)
    while _cost(c) > most:
        for size in ("B", "T"):
            if _cost(c) > most and c[size] > 1:
                c[size] = c[size] * 2 // 3
    return c


def work(case):
    e, B, T = 2 if case["dtype"] == "bf16" else 4, case["B"], case["T"]
    if case["op"].startswith("norm"):
        rows, D, R = B * T * (case["Hq"] + case["Hk"]), case["D"], case["R"]
        tables = 4 * T * R + (4 * B * T if case["positions"] else 0) + 8 * D
        if case["op"] == "norm":
            return {"bytes": 2 * e * rows * D + tables, "flops": rows * (4 * D + 3 * R)}
        return {"bytes": 4 * e * rows * D + tables + 8 * D, "flops": rows * (13 * D + 6 * R)}
    Hk, Hv, Dk, Dv = (case[n] for n in ("Hk", "Hv", "Dk", "Dv"))
    tokens = _lengths(case, 0)[1] if case["ragged"] else B * T
    qk, v, gates, state = 2 * e * tokens * Hk * Dk, e * tokens * Hv * Dv, 8 * tokens * Hv, 4 * B * Hv * Dk * Dv
    out = e * B * T * Hv * Dv
    if case["op"] == "step":
        return {"bytes": qk + v + gates + out + 2 * state, "flops": 7 * tokens * Hv * Dk * Dv}
    first = state if case["state"] else 0
    if case["op"] == "rule":
        return {"bytes": qk + v + gates + out + first + state, "flops": 7 * tokens * Hv * Dk * Dv}
    grads = 2 * e * B * T * Hk * Dk + e * B * T * Hv * Dv + 8 * B * T * Hv + first
    return {"bytes": qk + v + gates + 2 * out + first + state + state + grads, "flops": 21 * tokens * Hv * Dk * Dv}


def _lengths(case, seed):
    """Trajectories' lengths: the first is whole, one is empty where there are enough; the same number of tokens for every seed."""
    B, T = case["B"], case["T"]
    n = [T] + [(b * 7919 + 3) % (T + 1) for b in range(1, B)]
    if B > 3:
        n[2] = 0
    k = 1 + seed % (B - 1) if B > 1 else 0
    return [n[0]] + n[1 + k:] + n[1:1 + k], sum(n)


def prepare(case, seed):
    dev, dtype = torch.device("cuda"), TYPES[case["dtype"]]
    gen = torch.Generator(dev).manual_seed(seed)
    B, T = case["B"], case["T"]

    def normal(*shape):
        return torch.randn(*shape, generator=gen, device=dev)

    s = {"case": case, "seed": seed}
    if case["op"].startswith("norm"):
        Hq, Hk, D, R = (case[n] for n in ("Hq", "Hk", "D", "R"))
        # queries and keys as one projection gives them: slices of the same rows
        qk = (normal(B, T, Hq + Hk, D) * torch.exp(0.5 * normal(1, 1, Hq + Hk, 1))).to(dtype)
        s["q"], s["k"] = qk[:, :, :Hq], qk[:, :, Hq:]
        s["wq"], s["wk"] = 1 + 0.1 * normal(D), 1 + 0.1 * normal(D)
        P = 2 * T
        turn = torch.arange(P, dtype=torch.float64, device=dev)[:, None] * 10000.0 ** (-torch.arange(R // 2, dtype=torch.float64, device=dev) / (R // 2))
        s["cos"], s["sin"] = torch.cos(turn).float(), torch.sin(turn).float()
        s["positions"] = torch.randint(0, P, (B, T), generator=gen, device=dev, dtype=torch.int32) if case["positions"] else None
        s["q_out"], s["k_out"] = torch.empty(B, T, Hq, D, dtype=dtype, device=dev), torch.empty(B, T, Hk, D, dtype=dtype, device=dev)
        if case["op"] == "norm_train":
            s["dq_out"], s["dk_out"] = normal(B, T, Hq, D).to(dtype), normal(B, T, Hk, D).to(dtype)
            s["dq"], s["dk"] = torch.empty_like(s["q_out"]), torch.empty_like(s["k_out"])
            s["dwq"], s["dwk"] = torch.empty_like(s["wq"]), torch.empty_like(s["wk"])
        return s

    Hk, Hv, Dk, Dv = (case[n] for n in ("Hk", "Hv", "Dk", "Dv"))

    def unit(x):
        return x / x.square().sum(-1, keepdim=True).sqrt()

    # keys of one head lean to one side, as those of smooth fields do; decays of heads from slow to fast; writes between none and whole
    s["q"] = unit(normal(B, T, Hk, Dk) + 0.5 * normal(1, 1, Hk, Dk)).to(dtype)
    s["k"] = unit(normal(B, T, Hk, Dk) + 0.5 * normal(1, 1, Hk, Dk)).to(dtype)
    s["v"] = normal(B, T, Hv, Dv).to(dtype)
    s["g"] = -torch.rand(Hv, generator=gen, device=dev) * torch.nn.functional.softplus(normal(B, T, Hv) - 2)
    s["beta"] = torch.sigmoid(normal(B, T, Hv))
    s["scale"] = Dk ** -0.5
    s["o"] = torch.empty_like(s["v"])
    if case["op"] == "step":
        slots = B + B // 2 + 1  # the pool holds trajectories that do not take part in this step too
        s["state"] = normal(slots, Hv, Dk, Dv)
        s["slots"] = torch.randperm(slots, generator=gen, device=dev)[:B].to(torch.int32)
        for n in ("q", "k", "v", "g", "beta", "o"):
            s[n] = s[n][:, 0].contiguous()
        return s
    s["lengths"] = None
    if case["ragged"]:
        s["lengths"] = torch.tensor(_lengths(case, seed)[0], dtype=torch.int32, device=dev)
        padding = torch.arange(T, device=dev)[None] >= s["lengths"][:, None]
        for n in ("q", "k", "v", "g", "beta"):  # what nobody wrote
            s[n][padding] = float("nan")
    s["initial"] = normal(B, Hv, Dk, Dv) if case["state"] else None
    s["final"] = torch.empty(B, Hv, Dk, Dv, device=dev)
    if case["op"] == "rule_train":
        s["do"] = normal(B, T, Hv, Dv).to(dtype)
        if case["ragged"]:
            s["do"][padding] = float("nan")
        s["dfinal"] = normal(B, Hv, Dk, Dv)
        for n in ("q", "k", "v", "g", "beta"):
            s["d" + n] = torch.empty_like(s[n])
        s["dinitial"] = torch.empty_like(s["initial"]) if case["state"] else None
    return s


def run(s):
    return (_run_own if own else _run_plain)(s)


# ---------------------------------------------------------------- the framework's entry points

def _run_own(s):
    from paper_2504_11681_amd import binding as tfno
    op = s["case"]["op"]
    if op.startswith("norm"):
        ways = {"positions": s["positions"], "eps": EPS, "interleaved": s["case"]["pairs"] == "neighbours"}
        tables = (s["wq"], s["wk"], s["cos"], s["sin"])
        tfno.head_norm_rope(s["q"], s["k"], *tables, s["q_out"], s["k_out"], **ways)
        if op == "norm":
            return s["q_out"], s["k_out"]
        tfno.head_norm_rope_backward(s["q"], s["k"], *tables, s["dq_out"], s["dk_out"], s["dq"], s["dk"], s["dwq"], s["dwk"], **ways)
        return tuple(s[n] for n in ("q_out", "k_out", "dq", "dk", "dwq", "dwk"))
    inputs = tuple(s[n] for n in ("q", "k", "v", "g", "beta"))
    if op == "step":
        tfno.gated_delta_rule_step(*inputs, s["state"], s["o"], slots=s["slots"], scale=s["scale"])
        return s["o"], s["state"]
    ways = {"scale": s["scale"], "initial_state": s["initial"], "lengths": s["lengths"]}
    if op == "rule":
        tfno.gated_delta_rule(*inputs, s["o"], final_state=s["final"], **ways)
        return s["o"], s["final"]
    tape = tfno.gated_delta_rule_tape(s["q"], s["v"])
    tfno.gated_delta_rule(*inputs, s["o"], final_state=s["final"], tape=tape, **ways)
    grads = tuple(s["d" + n] for n in ("q", "k", "v", "g", "beta"))
    tfno.gated_delta_rule_backward(*inputs, s["do"], *grads, tape, d_final_state=s["dfinal"], d_initial_state=s["dinitial"], **ways)
    return (s["o"], s["final"], *grads) + ((s["dinitial"],) if s["dinitial"] is not None else ())


# ---------------------------------------------------------------- the plain forms

def _run_plain(s):
    op = s["case"]["op"]
    if op == "norm":
        return _plain_norm(s, s["q"], s["wq"]), _plain_norm(s, s["k"], s["wk"])
    if op == "norm_train":
        x = [s[n].detach().requires_grad_() for n in ("q", "k", "wq", "wk")]
        y = _plain_norm(s, x[0], x[2]), _plain_norm(s, x[1], x[3])
        d = torch.autograd.grad(y, x, (s["dq_out"], s["dk_out"]))
        return (y[0].detach(), y[1].detach(), *d)
    if op == "step":
        return _plain_step(s)
    if op == "rule":
        return _plain_rule(s, s["q"], s["k"], s["v"], s["g"], s["beta"], s["initial"])
    x = [s[n].detach().requires_grad_() for n in ("q", "k", "v", "g", "beta")]
    if s["initial"] is not None:
        x.append(s["initial"].detach().requires_grad_())
    o, final = _plain_rule(s, *x[:5], x[5] if len(x) > 5 else None)
    d = torch.autograd.grad((o, final), x, (_kept(s, s["do"]), s["dfinal"]))
    return (o.detach(), final.detach(), *d)


def _plain_norm(s, x, w):
    """x / sqrt(mean x^2 + eps) * w, its first R values rotated in pairs by the angle of their position."""
    R, f = s["case"]["R"], x.float()
    n = f * torch.rsqrt(f.square().mean(-1, keepdim=True) + EPS) * w
    at = slice(0, x.shape[1]) if s["positions"] is None else s["positions"].long()
    c, i = s["cos"][at].unsqueeze(-2), s["sin"][at].unsqueeze(-2)
    if s["case"]["pairs"] == "neighbours":
        a, b = n[..., 0:R:2], n[..., 1:R:2]
        turned = torch.stack((a * c - b * i, a * i + b * c), -1).flatten(-2)
    else:
        a, b = n[..., : R // 2], n[..., R // 2: R]
        turned = torch.cat((a * c - b * i, a * i + b * c), -1)
    return torch.cat((turned, n[..., R:]), -1).to(x.dtype)


def _plain_step(s):
    group = s["case"]["Hv"] // s["case"]["Hk"]
    q, k = (s[n].float().repeat_interleave(group, 1) for n in ("q", "k"))
    slots = s["slots"].long()
    S = s["state"][slots] * torch.exp(s["g"])[..., None, None]
    u = s["beta"][..., None] * (s["v"].float() - torch.matmul(k.unsqueeze(-2), S).squeeze(-2))
    S = S + k[..., None] * u[..., None, :]
    s["state"][slots] = S
    return (s["scale"] * torch.matmul(q.unsqueeze(-2), S).squeeze(-2)).to(s["o"].dtype), s["state"]


def _kept(s, x):
    """x with zeros where a trajectory has ended."""
    if s["lengths"] is None:
        return x
    live = torch.arange(x.shape[1], device=x.device)[None] < s["lengths"][:, None]
    return torch.where(live.reshape(live.shape + (1,) * (x.dim() - 2)), x, torch.zeros((), dtype=x.dtype, device=x.device))


def _inverse(N):
    """(I + N)^-1 of strictly lower triangular matrices of a power of two of rows: inverses of blocks on the diagonal, joined in pairs."""
    L, inv = N.shape[-1], torch.ones(*N.shape[:-1], 1, 1, device=N.device)
    for size in (2 ** p for p in range(L.bit_length() - 1)):
        m = L // (2 * size)
        pairs = torch.diagonal(N.unflatten(-1, (m, 2 * size)).unflatten(-3, (m, 2 * size)), dim1=-4, dim2=-2).movedim(-1, -3)
        upper, lower = inv[..., 0::2, :, :], inv[..., 1::2, :, :]
        corner = -torch.matmul(torch.matmul(lower, pairs[..., size:, :size]), upper)
        inv = torch.cat((torch.cat((upper, torch.zeros_like(upper)), -1), torch.cat((corner, lower), -1)), -2)
    return inv.squeeze(-3)


def _plain_rule(s, q, k, v, g, beta, initial):
    """The rule by chunks of up to 64 tokens.  With a chunk's incoming state S, G the running sum of g, M_ij = exp(G_i - G_j) for j <= i and
    T = (I + beta strict(M . K K'))^-1: U = T beta (V - e^G K S), O = scale (e^G Q S + (M . Q K') U), S' = e^GL S + (e^(GL-G) K)' U.
    The chunks depend on each other through S alone: everything else is done for all of them at once."""
    B, T, Hv, Dv = v.shape
    dtype, L = v.dtype, min(64, 1 << (T - 1).bit_length())
    n = -(-T // L)

    def chunks(x, heads):  # [B, T, H, D] -> [B, Hv, n, L, D]
        x = torch.nn.functional.pad(_kept(s, x).float(), (0, 0, 0, 0, 0, n * L - T))
        return x.repeat_interleave(heads, 2).transpose(1, 2).reshape(B, Hv, n, L, x.shape[-1])

    group = Hv // q.shape[2]
    q, k, v = chunks(q, group), chunks(k, group), chunks(v, 1)
    g, beta = chunks(g[..., None], 1).squeeze(-1), chunks(beta[..., None], 1)
    G = torch.cumsum(g, -1)
    lower = torch.ones(L, L, dtype=torch.bool, device=q.device).tril()
    M = torch.exp(torch.where(lower, G[..., :, None] - G[..., None, :], torch.full((), -math.inf, device=q.device)))
    G = G[..., None]
    kt = k.transpose(-1, -2).contiguous()
    Tb = _inverse((beta * M * torch.matmul(k, kt)).tril(-1)) * beta.transpose(-1, -2)
    P = M * torch.matmul(q, kt)
    W, U0 = torch.matmul(Tb, torch.exp(G) * k), torch.matmul(Tb, v)
    last = G[..., -1:, :]
    out_of = (torch.exp(last - G) * k).transpose(-1, -2).contiguous()
    S = torch.zeros(B, Hv, k.shape[-1], Dv, device=q.device) if initial is None else initial
    states, Us = [], []
    for c in range(n):
        U = U0[:, :, c] - torch.matmul(W[:, :, c], S)
        states.append(S)
        Us.append(U)
        S = torch.exp(last[:, :, c]) * S + torch.matmul(out_of[:, :, c], U)
    o = s["scale"] * (torch.exp(G) * torch.matmul(q, torch.stack(states, 2)) + torch.matmul(P, torch.stack(Us, 2)))
    return _kept(s, o.reshape(B, Hv, n * L, Dv)[:, :, :T].transpose(1, 2)).to(dtype), S


# ---------------------------------------------------------------- the definitions in 64 bits

def exact(case, seed):
    s = prepare(case, seed)
    if case["op"].startswith("norm"):
        q, k = _exact_norm(s, s["q"], s["wq"], s.get("dq_out")), _exact_norm(s, s["k"], s["wk"], s.get("dk_out"))
        return (q[0], k[0]) if case["op"] == "norm" else (q[0], k[0], q[1], k[1], q[2], k[2])
    if case["op"] == "step":
        slots = s["slots"].long()
        state = s["state"].double()
        o, S, _ = _exact_tokens(s, {n: _heads(s, s[n][:, None]) for n in ("q", "k", "v", "g", "beta")}, state[slots].flatten(0, 1))
        state[slots] = S.view(state[slots].shape)
        return o[0].view(s["o"].shape), state
    return _exact_rule(s)


def _exact_norm(s, x, w, dy):
    case, x, w = s["case"], x.double(), w.double()
    R, D = case["R"], case["D"]
    r = (x.square().sum(-1, keepdim=True) / D + EPS) ** -0.5
    at = torch.arange(case["T"], device=x.device).expand(case["B"], -1) if s["positions"] is None else s["positions"].long()
    c, i = s["cos"].double()[at][:, :, None], s["sin"].double()[at][:, :, None]
    pairs = torch.arange(R, device=x.device).view(-1, 2).t() if case["pairs"] == "neighbours" else torch.arange(R, device=x.device).view(2, -1)

    def turn(z, sign):
        out, a, b = z.clone(), z[..., pairs[0]], z[..., pairs[1]]
        out[..., pairs[0]], out[..., pairs[1]] = a * c - sign * b * i, b * c + sign * a * i
        return out

    y = turn(x * r * w, 1)
    if dy is None:
        return (y,)
    a = turn(dy.double(), -1)
    dn = a * w
    return y, r * dn - x * r ** 3 * (dn * x).sum(-1, keepdim=True) / D, (a * x * r).sum((0, 1, 2))


def _heads(s, x):
    """[B, T, H(, D)] in 64 bits as [T, B Hv(, D)], zeros past a trajectory's end."""
    x = _kept(s, x.double()) if s.get("lengths") is not None else x.double()
    return x.repeat_interleave(s["case"]["Hv"] // x.shape[2], 2).transpose(0, 1).flatten(1, 2).contiguous()


def _exact_tokens(s, x, S, first=0, count=None, keep=False):
    """Tokens one by one from state S: their outputs, the state after them, and if asked the states before each."""
    o, before = [], []
    for t in range(first, x["q"].shape[0] if count is None else first + count):
        if keep:
            before.append(S)
        Sb = S * torch.exp(x["g"][t])[:, None, None]
        u = x["beta"][t][:, None] * (x["v"][t] - torch.bmm(x["k"][t][:, None], Sb)[:, 0])
        S = torch.baddbmm(Sb, x["k"][t][:, :, None], u[:, None])
        if not keep:
            o.append(s["scale"] * torch.bmm(x["q"][t][:, None], S)[:, 0])
    return o, S, before


def _exact_rule(s):
    case = s["case"]
    B, T, Hk, Hv, Dk, Dv = (case[n] for n in ("B", "T", "Hk", "Hv", "Dk", "Dv"))
    if T * max(40e-6 if case["op"] == "rule" else 250e-6, B * Hv * Dk * Dv * 8 * (8 if case["op"] == "rule" else 40) / 2e12) > 20:
        return None
    x = {n: _heads(s, s[n]) for n in ("q", "k", "v", "g", "beta")}
    S = torch.zeros(B * Hv, Dk, Dv, dtype=torch.float64, device="cuda") if s["initial"] is None else s["initial"].double().flatten(0, 1)
    block = max(1, math.isqrt(T))
    o, at = [], []
    for first in range(0, T, block):
        at.append(S)
        some, S, _ = _exact_tokens(s, x, S, first, min(block, T - first))
        o += some

    def back(values):  # [T][B Hv, D...] -> [B, T, Hv, D...]
        v = torch.stack(values)
        return v.unflatten(1, (B, Hv)).transpose(0, 1)

    result = back(o), S.view(B, Hv, Dk, Dv)
    if case["op"] == "rule":
        return result
    do, dS = s["scale"] * _heads(s, s["do"]), s["dfinal"].double().flatten(0, 1)
    d = {n: [None] * T for n in x}
    for first in reversed(range(0, T, block)):
        count = min(block, T - first)
        before = _exact_tokens(s, x, at.pop(), first, count, keep=True)[2]
        for t in reversed(range(first, first + count)):
            q, k, v, beta, a = x["q"][t], x["k"][t], x["v"][t], x["beta"][t][:, None], torch.exp(x["g"][t])[:, None, None]
            Sb = before.pop() * a
            e = v - torch.bmm(k[:, None], Sb)[:, 0]
            St = torch.baddbmm(Sb, k[:, :, None], (beta * e)[:, None])
            d["q"][t] = torch.bmm(St, do[t][:, :, None])[:, :, 0]
            dS = torch.baddbmm(dS, q[:, :, None], do[t][:, None])
            du = torch.bmm(k[:, None], dS)[:, 0]
            de = beta * du
            d["k"][t] = torch.bmm(dS, (beta * e)[:, :, None])[:, :, 0] - torch.bmm(Sb, de[:, :, None])[:, :, 0]
            d["v"][t], d["beta"][t] = de, (du * e).sum(-1)
            dS = torch.baddbmm(dS, k[:, :, None], -de[:, None])
            d["g"][t] = (dS * Sb).sum((1, 2))
            dS = dS * a
    grads = {n: _kept(s, back(v)) for n, v in d.items()}
    for n in ("q", "k"):
        grads[n] = grads[n].unflatten(2, (Hk, Hv // Hk)).sum(3)
    return (*result, *(grads[n] for n in ("q", "k", "v", "g", "beta"))) + ((dS.view(B, Hv, Dk, Dv),) if s["initial"] is not None else ())
