"""The operators that a block along time is built and trained with: the gated linear recurrence (a state for each channel: whole sequences, their
gradient, one token at a time), the norms after one block and before the next with the gate and the residual between them (and their gradient), and
the norm over all gradients with the clipping to it.

``listed`` and ``draw`` give cases, ``prepare`` their inputs on the GPU, ``run`` one pass: with ``own`` false in elementary torch
operations in 32 bits, with ``own`` true through the framework's entry points.  ``exact`` gives the same in 64 bits from the
definition; ``work`` what a pass cannot do without.
"""
import math

import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
EPS = 1e-6


def listed():
    return [
        # one frame of one trajectory in a rollout, where latency counts
        _recurrence("recurrence step one", "step", "bf16", B=1, T=1, C=512),
        # a serving step of many trajectories out of a larger pool of states
        _recurrence("recurrence step many", "step", "bf16", B=512, T=1, C=4096),
        # pencils of 1024 points of a batch of 256 with 128 channels, read as sequences
        _recurrence("recurrence batch bf16", "recurrence", "bf16", B=256, T=1024, C=128),
        # one long trajectory with few channels, decays given as they are, from a state that an earlier part left
        _recurrence("recurrence long bf16", "recurrence", "bf16", B=1, T=16384, C=512, gates="decay", state=True),
        # training: both gates, the input scaled by what the decay leaves
        _recurrence("recurrence train bf16", "recurrence_train", "bf16", B=4, T=2048, C=2048),
        # training on float32 fields of odd sizes, trajectories of different lengths, a learned first state
        _recurrence("recurrence train odd f32", "recurrence_train", "f32", B=5, T=777, C=205, ragged=True, state=True),
        # one token between two blocks, residual stream in float32
        _norm("norms one token", "norms", "bf16", B=1, T=1, C=1024, gate="channel", residual="f32"),
        # a training batch between two blocks: a gate for each trajectory from its parameters, residual stream in float32
        _norm("norms train bf16", "norms_train", "bf16", B=16, T=1024, C=2048, gate="sequence", residual="f32"),
        # outputs of heads on their way to the projection: a norm for each head and a gate for each value, no residual; [tokens, heads, values]
        _norm("norms of heads train bf16", "norms_train", "bf16", B=8192, T=16, C=128, gate="token", activation="silu", residual="none", before=False),
        # float32 fields of odd sizes, trajectories of different lengths, a learned scale for each channel
        _norm("norms train odd f32", "norms_train", "f32", B=7, T=333, C=205, gate="channel", residual="f32", ragged=True),
        # the gradients of a small model
        _clip("clip small f32", [("f32", n) for n in (128 * 128, 128 * 128, 128 * 256, 8 * 128, 8, 256 * 256, 256, 128 * 256, 64, 64)]),
        # those of a large one: matrices in BF16, weights of norms in float32, sizes that are no multiple of anything
        _clip("clip large", [t for i in range(12) for t in (("bf16", 8192 * 2048), ("bf16", 2048 * 2048), ("bf16", 2048 * 133 + i), ("f32", 2048), ("f32", 205 + i))]),
    ]


def _recurrence(name, op, dtype, B, T, C, gates="both", ragged=False, state=False):
    c = {"op": op, "dtype": dtype, "B": B, "T": T, "C": C, "gates": gates, "ragged": ragged, "state": state}
    return {"name": name, **c} if name else c


def _norm(name, op, dtype, B, T, C, gate, residual, activation="none", after=True, before=True, ragged=False):
    c = {"op": op, "dtype": dtype, "B": B, "T": T, "C": C, "gate": gate, "activation": activation, "residual": residual, "after": after, "before": before,
         "ragged": ragged}
    return {"name": name, **c} if name else c


def _clip(name, tensors):
    # a case is plain values: "type:elements" of each tensor
    c = {"op": "clip", "dtype": "bf16" if any(t == "bf16" for t, _ in tensors) else "f32", "tensors": " ".join(f"{t}:{n}" for t, n in tensors)}
    return {"name": name, **c} if name else c


def _log(rng, low, high):
    return max(low, min(high, round(math.exp(rng.uniform(math.log(low), math.log(high))))))


def draw(rng):
    op = rng.choice(("step", "recurrence", "recurrence", "recurrence_train", "recurrence_train", "norms", "norms_train", "norms_train", "clip"))
    dtype = rng.choice(("f32", "bf16"))
    if op == "clip":
        most = max(_elements(c) for c in listed() if c["op"] == op)
        tensors = [(rng.choice(("f32", "bf16")), _log(rng, 1, 1 << 24)) for _ in range(_log(rng, 1, 60))]
        while sum(n for _, n in tensors) > most:
            tensors.pop()
        return _clip("", tensors)
    kind = op.split("_")[0]
    most = max(_elements(c) for c in listed() if c["op"].split("_")[0] == kind)
    if kind == "norms":
        c = _norm("", op, dtype, B=_log(rng, 1, 256), T=_log(rng, 1, 2048), C=rng.choice((_log(rng, 1, 8192), 64, 128, 512, 1024, 2048)),
                  gate=rng.choice(("none", "channel", "sequence", "token")), activation=rng.choice(("none", "silu", "sigmoid")),
                  residual=rng.choice(("none", "f32", dtype)), after=rng.random() < 0.75, before=rng.random() < 0.75, ragged=rng.random() < 0.3)
    else:
        c = _recurrence("", op, dtype, B=_log(rng, 1, 512), T=1 if op == "step" else _log(rng, 1, 16384), C=rng.choice((_log(rng, 1, 4096), 128, 512, 1024, 2048)),
                        gates=rng.choice(("both", "both", "one", "decay")), ragged=op != "step" and rng.random() < 0.3, state=op != "step" and rng.random() < 0.5)
    while _elements(c) > most:
        for size in ("B", "T"):
            if _elements(c) > most and c[size] > 1:
                c[size] = max(1, c[size] * 2 // 3)
    return c


def _tensors(case):
    return [(t, int(n)) for t, n in (x.split(":") for x in case["tensors"].split())]


def _elements(case):
    if case["op"] == "clip":
        return sum(n for _, n in _tensors(case))
    return case["B"] * case["T"] * case["C"]


def work(case):
    op = case["op"]
    size = {"f32": 4, "bf16": 2, "none": 0}
    e = size[case["dtype"]]
    if op == "clip":
        return {"bytes": sum(2 * size[t] * n for t, n in _tensors(case)), "flops": 3 * _elements(case)}
    B, T, C = case["B"], case["T"], case["C"]
    out, train = B * T * C, op.endswith("train")
    read = sum(_lengths(case, 0)) * C if case["ragged"] else out
    if op.startswith("norms"):
        r, token = size[case["residual"]], case["gate"] == "token"
        results = (0 if case["residual"] == "none" and case["before"] else r or e) + (e if case["before"] else 0)      # of r_out, n_out
        few = 4 * C * {"none": 0, "channel": 1, "sequence": B, "token": 0}[case["gate"]] + 4 * C * (case["after"] + case["before"])
        bytes_ = read * (e + r + token * e) + out * results + few
        if train:
            bytes_ += read * results + out * (e + r + token * e) + few
        return {"bytes": bytes_, "flops": read * (40 if train else 10)}
    inputs = {"both": 3, "one": 2, "decay": 2}[case["gates"]]
    state = 4 * B * C
    bytes_ = e * (inputs * read + out) + (2 * state if op == "step" else state + (state if case["state"] else 0))
    if train:
        bytes_ += e * (read + inputs * out) + state + (state if case["state"] else 0)
    return {"bytes": bytes_, "flops": read * (40 if train else 15)}


def _lengths(case, seed):
    """Trajectories' lengths: the first is whole, one is empty where there are enough; the same number of tokens for every seed."""
    B, T = case["B"], case["T"]
    n = [T] + [(b * 7919 + 3) % (T + 1) for b in range(1, B)]
    if B > 3:
        n[2] = 0
    k = 1 + seed % (B - 1) if B > 1 else 0
    return [n[0]] + n[1 + k:] + n[1:1 + k]


def prepare(case, seed):
    dev, dtype, op = torch.device("cuda"), TYPES[case["dtype"]], case["op"]
    gen = torch.Generator(dev).manual_seed(seed)

    def normal(*shape):
        return torch.randn(*shape, generator=gen, device=dev)

    s = {"case": case, "seed": seed}
    if op == "clip":
        # gradients of layers differ in size by orders of magnitude
        s["grads"] = [(normal(n) * 10.0 ** -(1 + i % 4)).to(TYPES[t]) for i, (t, n) in enumerate(_tensors(case))]
        s["norm"] = torch.empty((), device=dev)
        s["limit"] = 0.5 * float(torch.stack([g.float().square().sum() for g in s["grads"]]).sum().sqrt())
        return s
    B, T, C = case["B"], case["T"], case["C"]
    s["lengths"] = None
    if case["ragged"]:
        s["lengths"] = torch.tensor(_lengths(case, seed), dtype=torch.int32, device=dev)
        padding = torch.arange(T, device=dev)[None] >= s["lengths"][:, None]

    def tokens(x):
        if case["ragged"]:
            x[padding] = float("nan")  # what nobody wrote
        return x

    if op.startswith("norms"):
        res = None if case["residual"] == "none" else TYPES[case["residual"]]
        s["y"] = tokens((normal(B, T, C) * torch.exp(0.5 * normal(B, T, 1))).to(dtype))
        s["r"] = None if res is None else tokens((2 * normal(B, T, C)).to(res))
        # a gate for each value comes as a slice of a wider projection
        s["gate"] = {"none": lambda: None, "channel": lambda: 0.5 + 0.1 * normal(C), "sequence": lambda: 0.5 * normal(B, C),
                     "token": lambda: tokens(normal(B, T, 2 * C).to(dtype))[:, :, C:]}[case["gate"]]()
        s["w_after"], s["w_before"] = (1 + 0.1 * normal(C) if case[n] else None for n in ("after", "before"))
        s["scale"] = 0.9 if res is not None else 1.0
        s["r_out"] = None if res is None and case["before"] else torch.empty(B, T, C, dtype=res or dtype, device=dev)
        s["n_out"] = torch.empty(B, T, C, dtype=dtype, device=dev) if case["before"] else None
        if op == "norms_train":
            for n in ("r_out", "n_out"):
                s["d_" + n] = None if s[n] is None else tokens(normal(B, T, C).to(s[n].dtype))
            for n in ("y", "r", "gate", "w_after", "w_before"):
                s["d" + n] = None if s[n] is None else torch.empty(s[n].shape, dtype=s[n].dtype, device=dev)
        return s

    # gates before their sigmoid as one projection gives them; rates of channels from slow to fast; decays given as they are from slow to fast too
    s["x"] = tokens(normal(B, T, C).to(dtype))
    s["rate"] = s["input_gate"] = None
    if case["gates"] == "decay":
        s["gate"] = tokens((-torch.exp(normal(C) * 1.5 - 3) * torch.rand(B, T, C, generator=gen, device=dev)).to(dtype))
    else:
        both = tokens(normal(B, T, 2 * C).to(dtype))
        s["gate"] = both[:, :, :C]
        s["rate"] = 8 * torch.nn.functional.softplus(1.5 * normal(C) - 3)
        if case["gates"] == "both":
            s["input_gate"] = both[:, :, C:]
    s["normalise"] = case["gates"] != "decay"
    s["y"] = torch.empty(B, T, C, dtype=dtype, device=dev)
    if op == "step":
        pool = B + B // 2 + 1  # the pool holds trajectories that do not take part in this step too
        s["state"] = normal(pool, C)
        s["slots"] = torch.randperm(pool, generator=gen, device=dev)[:B].to(torch.int32)
        for n in ("x", "gate", "input_gate", "y"):
            s[n] = None if s[n] is None else s[n][:, 0]
        return s
    s["initial"] = normal(B, C) if case["state"] else None
    s["final"] = torch.empty(B, C, device=dev)
    if op == "recurrence_train":
        s["dy"], s["dfinal"] = tokens(normal(B, T, C).to(dtype)), normal(B, C)
        for n in ("x", "gate", "input_gate", "rate", "initial"):
            s["d" + n] = None if s[n] is None else torch.empty(s[n].shape, dtype=s[n].dtype, device=dev)
    return s


def run(s):
    return (_run_own if own else _run_plain)(s)


# ---------------------------------------------------------------- the framework's entry points

def _there(*tensors):
    return tuple(t for t in tensors if t is not None)


def _run_own(s):
    from paper_2504_11681_amd import binding as tfno
    op = s["case"]["op"]
    if op == "clip":
        tfno.clip_grad_norm(s["grads"], _limit(s), s["norm"])
        return (s["norm"], *s["grads"])
    if op.startswith("norms"):
        inputs = tuple(s[n] for n in ("y", "r", "gate", "w_after", "w_before"))
        ways = {"norm_after": s["case"]["after"], "activation": s["case"]["activation"], "residual_scale": s["scale"], "eps": EPS, "lengths": s["lengths"]}
        tfno.block_norm(*inputs, s["r_out"], s["n_out"], **ways)
        if op == "norms":
            return _there(s["r_out"], s["n_out"])
        grads = tuple(s["d" + n] for n in ("y", "r", "gate", "w_after", "w_before"))
        tfno.block_norm_backward(*inputs, s["d_r_out"], s["d_n_out"], *grads, **ways)
        return _there(s["r_out"], s["n_out"], *grads)
    inputs = tuple(s[n] for n in ("x", "gate", "input_gate", "rate"))
    if op == "step":
        tfno.gated_recurrence_step(*inputs, s["state"], s["y"], normalise=s["normalise"], slots=s["slots"])
        return s["y"], s["state"]
    ways = {"normalise": s["normalise"], "lengths": s["lengths"]}
    tape = tfno.gated_recurrence_tape(s["x"]) if op == "recurrence_train" else None
    tfno.gated_recurrence(*inputs, s["y"], initial_state=s["initial"], final_state=s["final"], tape=tape, **ways)
    if op == "recurrence":
        return s["y"], s["final"]
    grads = tuple(s["d" + n] for n in ("x", "gate", "input_gate", "rate"))
    tfno.gated_recurrence_backward(*inputs, s["dy"], *grads, tape, d_final_state=s["dfinal"], d_initial_state=s["dinitial"], **ways)
    return _there(s["y"], s["final"], *grads, s["dinitial"])


# ---------------------------------------------------------------- the plain forms

def _limit(s):
    """The limit of this pass: a little lower than that of the one before, so that every pass has something to clip."""
    limit = s["limit"]
    s["limit"] = 0.999 * limit
    return limit


def _run_plain(s):
    op = s["case"]["op"]
    if op == "clip":
        return _plain_clip(s)
    if op == "step":
        return _plain_step(s)
    norms = op.startswith("norms")
    names = ("y", "r", "gate", "w_after", "w_before") if norms else ("x", "gate", "input_gate", "rate", "initial")
    x = {n: s[n] for n in names}
    if not op.endswith("train"):
        return _there(*(_plain_norms if norms else _plain_recurrence)(s, **x))
    x = {n: None if t is None else t.detach().requires_grad_() for n, t in x.items()}
    out = (_plain_norms if norms else _plain_recurrence)(s, **x)
    d = (s["d_r_out"], s["d_n_out"]) if norms else (s["dy"], s["dfinal"])
    d = [t if t is s.get("dfinal") else _kept(s, t) for t in d]
    pairs = [(o, t) for o, t in zip(out, d) if o is not None]
    grads = torch.autograd.grad([o for o, _ in pairs], _there(*x.values()), [t for _, t in pairs])
    return (*(o.detach() for o, _ in pairs), *grads)


def _kept(s, x):
    """x[B, T, C] with zeros where a trajectory has ended."""
    if x is None or s["lengths"] is None:
        return x
    live = torch.arange(x.shape[1], device=x.device)[None] < s["lengths"][:, None]
    return torch.where(live[..., None], x, torch.zeros((), dtype=x.dtype, device=x.device))


def _plain_clip(s):
    limit = _limit(s)
    norm = torch.stack([g.float().square().sum() for g in s["grads"]]).sum().sqrt()
    scale = torch.where(norm > limit, limit / norm, torch.ones_like(norm))
    for g in s["grads"]:
        g.copy_(g.float() * scale)
    s["norm"].copy_(norm)
    return (s["norm"], *s["grads"])


def _plain_norms(s, y, r, gate, w_after, w_before):
    """r_out = scale r + act(gate) Norm(y) w_after, n_out = Norm(r_out) w_before."""
    case = s["case"]
    dtype, m = y.dtype, _kept(s, y).float()
    if case["after"]:
        m = m * torch.rsqrt(m.square().mean(-1, keepdim=True) + EPS) * w_after
    if gate is not None:
        z = (_kept(s, gate) if case["gate"] == "token" else gate[:, None] if case["gate"] == "sequence" else gate).float()
        if case["activation"] != "none":
            z = (z if case["activation"] == "silu" else 1.0) / (1.0 + torch.exp(-z))
        m = m * z
    if r is not None:
        m = m + s["scale"] * _kept(s, r).float()
    n = None
    if case["before"]:
        n = _kept(s, (m * torch.rsqrt(m.square().mean(-1, keepdim=True) + EPS) * w_before).to(dtype))
    return None if s["r_out"] is None else _kept(s, m.to(s["r_out"].dtype)), n


def _plain_gates(s, x, gate, input_gate, rate):
    """Decays of tokens and what each adds to the state."""
    log = gate.float() if rate is None else -rate / (1.0 + torch.exp(-gate.float()))
    u = x.float()
    if input_gate is not None:
        u = u / (1.0 + torch.exp(-input_gate.float()))
    if s["normalise"]:
        u = u * torch.sqrt(-torch.expm1(2 * log))
    return torch.exp(log), u


def _plain_step(s):
    slots = s["slots"].long()
    a, u = _plain_gates(s, s["x"], s["gate"], s["input_gate"], s["rate"])
    h = a * s["state"][slots] + u
    s["state"][slots] = h
    return h.to(s["y"].dtype), s["state"]


def _plain_recurrence(s, x, gate, input_gate, rate, initial):
    """h = a h + u for all tokens: each takes in the 1, 2, 4, ... tokens before it."""
    dtype, T = x.dtype, x.shape[1]
    a, u = _plain_gates(s, *(_kept(s, t) for t in (x, gate, input_gate)), rate)
    if s["lengths"] is not None:  # past a trajectory's end the state stays
        live = (torch.arange(T, device=x.device)[None] < s["lengths"][:, None])[..., None]
        a, u = torch.where(live, a, torch.ones_like(a)), torch.where(live, u, torch.zeros_like(u))
    if initial is not None:
        u = torch.cat((u[:, :1] + a[:, :1] * initial[:, None], u[:, 1:]), 1)
    step = 1
    while step < T:
        u = torch.cat((u[:, :step], u[:, step:] + a[:, step:] * u[:, :-step]), 1)
        a = torch.cat((a[:, :step], a[:, step:] * a[:, :-step]), 1)
        step *= 2
    return _kept(s, u.to(dtype)), u[:, -1]


# ---------------------------------------------------------------- the definitions in 64 bits

def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "clip":
        norm = math.sqrt(math.fsum(float((g.double() ** 2).sum()) for g in s["grads"]))
        return (torch.tensor(norm, dtype=torch.float64, device="cuda"), *(g.double() * min(1.0, s["limit"] / norm) for g in s["grads"]))
    if op.startswith("norms"):
        return _exact_norms(s)
    if op == "step":
        slots, state = s["slots"].long(), s["state"].double()
        a, u = _exact_gates(s, *(None if s[n] is None else s[n].double() for n in ("x", "gate", "input_gate", "rate")))[:2]
        state[slots] = a * state[slots] + u
        return state[slots], state
    return _exact_recurrence(s)


def _exact_gates(s, x, gate, input_gate, rate):
    sigma = None if rate is None else torch.special.expit(gate)
    log = gate if rate is None else -rate * sigma
    opened = torch.ones_like(x) if input_gate is None else torch.special.expit(input_gate)
    left = (-torch.special.expm1(2 * log)) ** 0.5 if s["normalise"] else torch.ones_like(x)
    return torch.special.exp2(log / math.log(2.0)), x * opened * left, log, sigma, opened, left


def _exact_recurrence(s):
    case = s["case"]
    B, T, C = (case[n] for n in ("B", "T", "C"))
    if T * 6e-5 + B * T * C * 8 * 60 / 2e12 > 20:
        return None
    x, gate, input_gate = ((None if s[n] is None else _kept(s, s[n].double())) for n in ("x", "gate", "input_gate"))
    rate = None if s["rate"] is None else s["rate"].double()
    a, u, log, sigma, opened, left = _exact_gates(s, x, gate, input_gate, rate)
    ends = [T] * B if s["lengths"] is None else s["lengths"].tolist()
    live = torch.tensor([[float(t < n) for t in range(T)] for n in ends], dtype=torch.float64, device="cuda")[..., None]
    a, u = a * live + (1 - live), u * live
    h = torch.zeros(B, C, dtype=torch.float64, device="cuda") if s["initial"] is None else s["initial"].double()
    before = torch.empty(B, T, C, dtype=torch.float64, device="cuda")
    y = torch.empty_like(before)
    for t in range(T):
        before[:, t] = h
        h = a[:, t] * h + u[:, t]
        y[:, t] = h
    if case["op"] == "recurrence":
        return y * live, h
    dy, d = _kept(s, s["dy"].double()), s["dfinal"].double()
    dh = torch.empty_like(before)  # of the state after each token
    for t in reversed(range(T)):
        d = d + dy[:, t]
        dh[:, t] = d
        d = a[:, t] * d
    dlog = dh * a * before * live
    du = dh * live
    dx = du * opened * left
    if s["normalise"]:  # left' = -exp(2 log) / left
        dlog = dlog - du * x * opened * a ** 2 / torch.where(left > 0, left, 1.0)
    grads = [dx, dlog if rate is None else -dlog * rate * sigma * (1 - sigma)]
    if input_gate is not None:
        grads.append(du * x * left * opened * (1 - opened))
    if rate is not None:
        grads.append(-(dlog * sigma).sum((0, 1)))
    return (y * live, h, *grads) + ((d,) if s["initial"] is not None else ())


def _exact_norms(s):
    case = s["case"]
    C = case["C"]
    y, r = _kept(s, s["y"].double()), None if s["r"] is None else _kept(s, s["r"].double())
    one = torch.ones((), dtype=torch.float64, device="cuda")
    root_y = (y.square().sum(-1, keepdim=True) / C + EPS) ** -0.5 if case["after"] else one
    w = s["w_after"].double() if case["after"] else one
    m = y * root_y * w
    z = None
    if s["gate"] is not None:
        z = {"token": lambda: _kept(s, s["gate"].double()), "sequence": lambda: s["gate"].double()[:, None].expand_as(y),
             "channel": lambda: s["gate"].double().expand_as(y)}[case["gate"]]()
    open_, slope = one, one
    if z is not None:
        sigma = torch.special.expit(z)
        open_ = {"none": z, "silu": z * sigma, "sigmoid": sigma}[case["activation"]]
        slope = {"none": torch.ones_like(z), "silu": sigma * (1 + z * (1 - sigma)), "sigmoid": sigma * (1 - sigma)}[case["activation"]]
    stream = open_ * m + (s["scale"] * r if r is not None else 0.0)
    root_s = (stream.square().sum(-1, keepdim=True) / C + EPS) ** -0.5
    out = [] if s["r_out"] is None else [_kept(s, stream)]
    if case["before"]:
        out.append(_kept(s, stream * root_s * s["w_before"].double()))
    if case["op"] == "norms":
        return tuple(out)
    d = torch.zeros_like(y) if s["d_r_out"] is None else _kept(s, s["d_r_out"].double())
    dw_before = None
    if case["before"]:
        dn = _kept(s, s["d_n_out"].double())
        dw_before = (dn * stream * root_s).sum((0, 1))
        dn = dn * s["w_before"].double()
        d = d + root_s * (dn - stream * root_s ** 2 * (dn * stream).sum(-1, keepdim=True) / C)
    dr = None if r is None else s["scale"] * d
    dgate = None
    if z is not None:
        dgate = d * m * slope
        dgate = {"token": lambda: dgate, "sequence": lambda: dgate.sum(1), "channel": lambda: dgate.sum((0, 1))}[case["gate"]]()
    dm = d * open_
    dw_after = None
    if case["after"]:
        dw_after = (dm * y * root_y).sum((0, 1))
        dm = dm * w
        dm = root_y * (dm - y * root_y ** 2 * (dm * y).sum(-1, keepdim=True) / C)
    return (*out, *_there(dm, dr, dgate, dw_after, dw_before))
