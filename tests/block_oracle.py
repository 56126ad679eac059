"""The operators of a block along time in float64 from their definitions, and how far float32 and BF16 results may be off.

Bounds, from the arithmetic: a BF16 result is rounded once, at most 2^-8 of each value.  A float32 result of the recurrence is a state that its tokens round one after the other,
2^-24 each of either sign, while it lasts: over n tokens sqrt(n) of them, 45 for the longest sequence here, with gates of some 4 roundings each; the norms are sums of up to 8192
squares in a tree and a handful of products: 64 * 2^-24 for both.  Gradients of gates are differences of two such values that cancel in part, those of weights sums over tokens that
do: four times that.  What goes into a BF16 result is that far off too."""
import torch

F32, BF16 = torch.float32, torch.bfloat16
REL = {BF16: 2.0 ** -8 + 2.0 ** -14, F32: 64 * 2.0 ** -24}
REL_SUMS = 256 * 2.0 ** -24
REL_GATES = {BF16: 2.0 ** -8 + 2.0 ** -14, F32: 256 * 2.0 ** -24}


def rel(got, want):
    assert got.shape == want.shape, (got.shape, want.shape)
    got, want = got.double(), want.double()
    assert torch.isfinite(got).all()
    off, norm = float((got - want).norm()), float(want.norm())
    return off / norm if norm else off


def live_of(lengths, B, T, device):
    if lengths is None:
        return torch.ones(B, T, 1, dtype=torch.bool, device=device)
    return (torch.arange(T, device=device)[None] < lengths.clamp(0, T)[:, None])[..., None]


def only(live, x):
    return None if x is None else torch.where(live, x.double(), torch.zeros((), dtype=torch.float64, device=live.device))


def recurrence(x, gate, input_gate, rate, normalise, initial=None, lengths=None, d_y=None, d_final=None):
    """y, final, and with d_y the gradients of x, gate, input_gate, rate and the initial state (None where there is none)."""
    B, T, C = x.shape
    live = live_of(lengths, B, T, x.device)
    x, gate, input_gate = (only(live, t) for t in (x, gate, input_gate))
    s = None if rate is None else torch.sigmoid(gate)
    l = gate if rate is None else -rate.double() * s
    a = l.exp()
    o = torch.ones_like(x) if input_gate is None else torch.sigmoid(input_gate)
    left = torch.sqrt(-torch.expm1(2 * l)) if normalise else torch.ones_like(x)
    h = torch.zeros(B, C, dtype=torch.float64, device=x.device) if initial is None else initial.double()
    before, y = [], torch.zeros_like(x)
    for t in range(T):
        before.append(h)
        h = torch.where(live[:, t], torch.where(a[:, t] == 0, 0.0, a[:, t] * h) + x[:, t] * o[:, t] * left[:, t], h)
        y[:, t] = torch.where(live[:, t], h, 0.0)
    if d_y is None:
        return y, h
    final, d_y = h, only(live, d_y)
    D = torch.zeros_like(h) if d_final is None else d_final.double()
    dx, dl, do = torch.zeros_like(x), torch.zeros_like(x), torch.zeros_like(x)
    for t in reversed(range(T)):
        at = live[:, t]
        G = D + d_y[:, t]
        dx[:, t] = torch.where(at, G * o[:, t] * left[:, t], 0.0)
        do[:, t] = torch.where(at, G * x[:, t] * left[:, t], 0.0)
        through = torch.where(a[:, t] == 0, 0.0, G * a[:, t] * before[t])
        if normalise:
            through = through - torch.where(left[:, t] == 0, 0.0, G * x[:, t] * o[:, t] * a[:, t] ** 2 / left[:, t])
        dl[:, t] = torch.where(at, through, 0.0)
        D = torch.where(at, torch.where(a[:, t] == 0, 0.0, a[:, t] * G), D)
    dgate = dl if rate is None else dl * -rate.double() * s * (1 - s)
    drate = None if rate is None else -(dl * s).sum((0, 1))
    return y, final, dx, dgate, None if input_gate is None else do * o * (1 - o), drate, D


def between(y, r, gate, w_after, w_before, norm_after, activation, scale, eps, lengths=None, d_r=None, d_n=None, results=(True, True)):
    """r_out, n_out, and with gradients of them those of y, r, gate, w_after, w_before (autograd in float64)."""
    B, T, C = y.shape
    live = live_of(lengths, B, T, y.device)
    x = [only(live, y), only(live, r), only(live, gate) if gate is not None and gate.dim() == 3 else None if gate is None else gate.double(),
         torch.ones(C, dtype=torch.float64, device=y.device) if w_after is None else w_after.double(),
         torch.ones(C, dtype=torch.float64, device=y.device) if w_before is None else w_before.double()]
    x = [None if t is None else t.detach().requires_grad_() for t in x]
    m = x[0]
    if norm_after:
        m = m / torch.sqrt((m * m).mean(-1, keepdim=True) + eps) * x[3]
    if gate is not None:
        z = x[2][:, None] if gate.dim() == 2 else x[2]
        m = m * {"none": lambda v: v, "silu": lambda v: v * torch.sigmoid(v), "sigmoid": torch.sigmoid}[activation](z)
    if r is not None:
        m = m + scale * x[1]
    n = m / torch.sqrt((m * m).mean(-1, keepdim=True) + eps) * x[4]
    out = [torch.where(live, t, 0.0) for t in (m, n)]
    if d_r is None and d_n is None:
        return tuple(t.detach() for t in out)
    total = sum((o * only(live, d)).sum() for o, d in zip(out, (d_r, d_n)) if d is not None)
    grads = torch.autograd.grad(total, [t for t in x if t is not None], allow_unused=True)
    grads = iter(grads)
    return tuple(t.detach() for t in out) + tuple(None if t is None else next(grads) for t in x)
