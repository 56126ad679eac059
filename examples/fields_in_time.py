"""Fields that move: a Fourier layer reads every frame, the gated delta rule carries what was seen, the next frame comes out.

Each sequence is a periodic field of a few waves that travel at a speed of the sequence's own and fade; a single frame does not tell that speed, the
frames before it do.  A frame u[N] goes through the Fourier layer of real fields (fno1d_real, with fixed random modes) and is sampled at a few points; queries, keys, values and
the two gates are linear in that, queries and keys are normalised and rotated (head_norm_rope), the rule (gated_delta_rule) mixes along time, and a
linear map gives the next frame's change.  Training runs whole sequences forward and backward; the rollout reads the first frames at once, keeps the
state and goes on token by token (gated_delta_rule_step) on its own predictions.  The maps and the optimiser are PyTorch's, the rest is the library's.

    python examples/fields_in_time.py --steps 200
"""
import argparse
import math
import os
import sys

import torch
import torch.nn.functional as F

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2504_11681_amd import binding as tfno  # noqa: E402


class HeadNormRope(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, wq, wk, cos, sin, positions):
        ctx.save_for_backward(q, k, wq, wk, cos, sin, positions)
        return tfno.head_norm_rope(q, k, wq, wk, cos, sin, torch.empty(q.shape, dtype=q.dtype, device=q.device),
                                   torch.empty(k.shape, dtype=k.dtype, device=k.device), positions)

    @staticmethod
    def backward(ctx, dq_out, dk_out):
        q, k, wq, wk, cos, sin, positions = ctx.saved_tensors
        dq, dk, dwq, dwk = (torch.empty(x.shape, dtype=x.dtype, device=x.device) for x in (q, k, wq, wk))
        tfno.head_norm_rope_backward(q, k, wq, wk, cos, sin, dq_out.contiguous(), dk_out.contiguous(), dq, dk, dwq, dwk, positions)
        return dq, dk, dwq, dwk, None, None, None


class GatedDeltaRule(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, v, g, beta):
        """Outputs and the state after the last token."""
        o = torch.empty(v.shape, dtype=v.dtype, device=v.device)
        final = torch.empty(v.shape[0], v.shape[2], k.shape[3], v.shape[3], device=v.device)
        tape = tfno.gated_delta_rule_tape(q, v) if any(ctx.needs_input_grad) else None
        tfno.gated_delta_rule(q, k, v, g, beta, o, final_state=final, tape=tape)
        if tape is not None:
            ctx.save_for_backward(q, k, v, g, beta, tape)
        return o, final

    @staticmethod
    def backward(ctx, d_o, d_final):
        q, k, v, g, beta, tape = ctx.saved_tensors
        d = [torch.empty(x.shape, dtype=x.dtype, device=x.device) for x in (q, k, v, g, beta)]
        tfno.gated_delta_rule_backward(q, k, v, g, beta, d_o.contiguous(), *d, tape, d_final_state=d_final.contiguous())
        return tuple(d)


class FieldsInTime(torch.nn.Module):
    """u[B, T, N] to the next frames; `dtype` is what queries, keys and values are held in."""

    def __init__(self, N=256, modes=24, channels=4, points=32, key_heads=2, heads=4, D=64, longest=512, dtype=torch.bfloat16):
        super().__init__()
        self.N, self.channels, self.points, self.key_heads, self.heads, self.D, self.dtype = N, channels, points, key_heads, heads, D, dtype
        seen = channels * points
        self.q, self.k = torch.nn.Linear(seen, key_heads * D, bias=False), torch.nn.Linear(seen, key_heads * D, bias=False)
        self.v, self.gates = torch.nn.Linear(seen, heads * D, bias=False), torch.nn.Linear(seen, 2 * heads)
        self.next, self.skip = torch.nn.Linear(heads * D, N), torch.nn.Linear(seen, N, bias=False)
        with torch.no_grad():                              # the change of a frame starts at zero
            self.next.weight.mul_(0.1), self.next.bias.zero_(), self.skip.weight.zero_()
        # keys of length one: the rule then replaces along a key and never overshoots
        self.wq, self.wk = torch.nn.Parameter(torch.ones(D)), torch.nn.Parameter(torch.full((D,), D ** -0.5))
        angle = torch.arange(longest)[:, None] * 100.0 ** (-torch.arange(D // 4) / (D // 4))[None]
        self.register_buffer("cos", angle.cos()), self.register_buffer("sin", angle.sin())
        self.register_buffer("modes", torch.randn(1, channels, modes, dtype=torch.complex64))     # features of a frame; not trained

    def see(self, u):
        """u[B, T, N] to samples of its Fourier layer [B, T, channels * points]."""
        B, T, N = u.shape
        y = torch.empty(B * T, self.channels, N, device=u.device)
        tfno.fno1d_real(u.reshape(B * T, 1, N).contiguous(), self.modes, y)
        return y[:, :, ::N // self.points].reshape(B, T, -1)

    def tokens(self, u, at):
        """What the rule takes for the frames u[B, T, N] at the positions at[B, T]."""
        h = self.see(u)
        q, k = (f(h).to(self.dtype).unflatten(-1, (self.key_heads, self.D)) for f in (self.q, self.k))
        q, k = HeadNormRope.apply(q, k, self.wq, self.wk, self.cos, self.sin, at)
        v = self.v(h).to(self.dtype).unflatten(-1, (self.heads, self.D))
        forget, write = self.gates(h).chunk(2, -1)
        return h, q, k, v, -0.1 * F.softplus(forget), torch.sigmoid(write).contiguous()

    def out(self, u, h, o):
        return u + self.next(o.float().flatten(2)) + self.skip(h)

    def forward(self, u):
        """The frames after u[B, T, N], and the state that a rollout goes on from."""
        B, T, _ = u.shape
        h, *x = self.tokens(u, torch.arange(T, dtype=torch.int32, device=u.device).expand(B, T).contiguous())
        o, state = GatedDeltaRule.apply(*x)
        return self.out(u, h, o), state

    @torch.no_grad()
    def step(self, u, t, state):
        """The frame after u[B, N], the frame of time t; advances the state."""
        B = u.shape[0]
        h, *x = self.tokens(u[:, None], torch.full((B, 1), t, dtype=torch.int32, device=u.device))
        q, k, v, g, beta = (y[:, 0] for y in x)
        o = torch.empty(v.shape, dtype=v.dtype, device=v.device)
        tfno.gated_delta_rule_step(q, k, v, g, beta, state, o)
        return self.out(u[:, None], h, o[:, None])[:, 0]


def fields(B, T, N, gen, waves=5):
    """u[B, T, N] float32: `waves` waves of 1 .. waves periods, all with the sequence's own speed and decay."""
    def uniform(low, high, *shape):
        return low + (high - low) * torch.rand(*shape, generator=gen, device=gen.device)

    j = torch.arange(1, waves + 1, device=gen.device)[None, :, None, None]
    x = torch.arange(N, device=gen.device)[None, None, None] / N
    t = torch.arange(T, device=gen.device)[None, None, :, None]
    speed, fade = uniform(-0.02, 0.02, B, 1, 1, 1), uniform(0.0, 0.01, B, 1, 1, 1)
    size, phase = uniform(0.3, 1.0, B, waves, 1, 1), uniform(0.0, 2 * math.pi, B, waves, 1, 1)
    return (size * torch.exp(-fade * t) * torch.sin(2 * math.pi * j * (x - speed * t) + phase)).sum(1)


def loss_of(model, u):
    """Squared error of the next frames over that of taking the frame before."""
    predicted, _ = model(u[:, :-1])
    return (predicted - u[:, 1:]).square().mean() / (u[:, 1:] - u[:, :-1]).square().mean()


def train(model, steps, B=16, T=129, lr=2e-3, seed=1, say=print):
    gen = torch.Generator("cuda").manual_seed(seed)
    optimizer = torch.optim.Adam(model.parameters(), lr=lr)
    slower = torch.optim.lr_scheduler.LambdaLR(optimizer, lambda i: 1.0 - i / steps)
    losses = []
    for i in range(steps):
        optimizer.zero_grad()
        loss = loss_of(model, fields(B, T, model.N, gen))
        loss.backward()
        optimizer.step()
        slower.step()
        losses.append(float(loss.detach()))
        if i % 20 == 0 or i + 1 == steps:
            say(f"step {i}: error of the next frame {losses[-1]:.4f} of that of the frame before", flush=True)
    return losses


@torch.no_grad()
def rollout(model, u, more):
    """`more` frames after u[B, T, N], each from the one before."""
    predicted, state = model(u)
    frames = [predicted[:, -1]]
    for t in range(u.shape[1], u.shape[1] + more - 1):
        frames.append(model.step(frames[-1], t, state))
    return torch.stack(frames, 1)


def main():
    parser = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    parser.add_argument("--steps", type=int, default=200)
    parser.add_argument("--more", type=int, default=16, help="frames of the rollout")
    a = parser.parse_args()
    torch.manual_seed(0)
    model = FieldsInTime().cuda()
    train(model, a.steps)
    u = fields(8, 128 + a.more, model.N, torch.Generator("cuda").manual_seed(2))
    frames, truth = rollout(model, u[:, :128], a.more), u[:, 128:]
    for n in sorted({1, a.more // 2, a.more} - {0}):
        still = (u[:, 127] - truth[:, n - 1]).norm() / truth[:, n - 1].norm()
        print(f"{n} frames on: off by {float((frames[:, n - 1] - truth[:, n - 1]).norm() / truth[:, n - 1].norm()):.3f}, the last frame seen by {float(still):.3f}")


if __name__ == "__main__":
    main()
