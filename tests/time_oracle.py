"""The operators along time in float64, token by token from their definitions, and how far float32 and BF16 results may be off.

Bounds, from the arithmetic: a BF16 result has 8 significant bits and is rounded once, at most 2^-8 of each value, so its L2 error is at most 2^-8 of
its norm; what it is rounded from carries two-part operands, 2^-15 at most.  Float32 results are sums of some hundred terms of either sign, each 2^-24 off, and
pass through a handful of such sums one after the other: 64 * 2^-24.  The gradient of the gates is a running sum of differences that cancel in part:
four times that."""
import torch

REL = {torch.bfloat16: 2.0 ** -8 + 2.0 ** -14, torch.float32: 64 * 2.0 ** -24}
REL_GATES = 256 * 2.0 ** -24


def rel(got, want):
    assert got.shape == want.shape, (got.shape, want.shape)
    got, want = got.double(), want.double()
    assert torch.isfinite(got).all()
    off, norm = float((got - want).norm()), float(want.norm())
    return off / norm if norm else off


def tokens_of(lengths, B, T, device):
    if lengths is None:
        return torch.ones(B, T, dtype=torch.bool, device=device)
    return torch.arange(T, device=device)[None] < lengths.clamp(0, T)[:, None]


def rule(q, k, v, g, beta, scale, initial=None, lengths=None, d_o=None, d_final=None):
    """o, final, and with d_o the gradients of q, k, v, g, beta and the initial state."""
    B, T, Hk, Dk = q.shape
    Hv, Dv = v.shape[2:]
    live = tokens_of(lengths, B, T, q.device)

    def f64(x, heads):
        if x is None:
            return torch.zeros(B, T, Hv, dtype=torch.float64, device=q.device)
        x = torch.where(live.reshape(B, T, *(1,) * (x.dim() - 2)), x.double(), torch.zeros((), dtype=torch.float64, device=q.device))
        return x.repeat_interleave(heads, 2)

    group = Hv // Hk
    q, k, v, g, beta = f64(q, group), f64(k, group), f64(v, 1), f64(g, 1), f64(beta, 1)
    S = torch.zeros(B, Hv, Dk, Dv, dtype=torch.float64, device=q.device) if initial is None else initial.double()
    states, o = [], torch.zeros(B, T, Hv, Dv, dtype=torch.float64, device=q.device)
    for t in range(T):
        states.append(S)
        Sb = S * g[:, t].exp()[..., None, None]
        u = beta[:, t, :, None] * (v[:, t] - (k[:, t, :, :, None] * Sb).sum(-2))
        S = Sb + k[:, t, :, :, None] * u[..., None, :]
        o[:, t] = scale * (q[:, t, :, :, None] * S).sum(-2)
    if d_o is None:
        return o, S
    final, d_o = S, f64(d_o, 1) * scale
    dS = torch.zeros_like(S) if d_final is None else d_final.double()
    d = {n: torch.zeros(x.shape, dtype=torch.float64, device=x.device) for n, x in (("q", q), ("k", k), ("v", v), ("g", g), ("beta", beta))}
    for t in reversed(range(T)):
        a, be, kt = g[:, t].exp()[..., None, None], beta[:, t, :, None], k[:, t]
        Sb = states[t] * a
        e = v[:, t] - (kt[..., None] * Sb).sum(-2)
        St = Sb + kt[..., None] * (be * e)[..., None, :]
        d["q"][:, t] = (St * d_o[:, t, :, None, :]).sum(-1)
        dS = dS + q[:, t, :, :, None] * d_o[:, t, :, None, :]
        du = (kt[..., None] * dS).sum(-2)
        de = be * du
        d["beta"][:, t] = (du * e).sum(-1)
        d["v"][:, t] = de
        d["k"][:, t] = (dS * (be * e)[..., None, :]).sum(-1) - (Sb * de[..., None, :]).sum(-1)
        dS = dS - kt[..., None] * de[..., None, :]
        d["g"][:, t] = (dS * Sb).sum((-1, -2)) * live[:, t, None]
        dS = dS * a
    for n in ("q", "k"):
        d[n] = d[n].unflatten(2, (Hk, group)).sum(3)
    return o, final, d["q"], d["k"], d["v"], d["g"], d["beta"], dS


def norm(x, w, cos, sin, positions, eps, interleaved, dy=None):
    """y, and with dy the gradients of x and w."""
    B, T, H, D = x.shape
    x = x.double()
    w = torch.ones(D, dtype=torch.float64, device=x.device) if w is None else w.double()
    r = 1.0 / torch.sqrt((x * x).mean(-1, keepdim=True) + eps)
    R = 0 if cos is None else 2 * cos.shape[1]
    i = torch.arange(R // 2, device=x.device)
    first, second = (2 * i, 2 * i + 1) if interleaved else (i, i + R // 2)
    if R:
        p = torch.arange(T, device=x.device).expand(B, T) if positions is None else positions.long()
        c, s = cos.double()[p][:, :, None], sin.double()[p][:, :, None]

    def turn(z, sign):
        z = z.clone()
        if R:
            a, b = z[..., first].clone(), z[..., second].clone()
            z[..., first], z[..., second] = a * c - sign * b * s, sign * a * s + b * c
        return z

    y = turn(x * r * w, 1.0)
    if dy is None:
        return y
    a = turn(dy.double(), -1.0)
    n = x * r
    return y, r * (a * w - n * (a * w * n).mean(-1, keepdim=True)), (a * n).sum((0, 1, 2))
