"""Fields that move, by blocks with a state for every channel: each block mixes along time (gated_recurrence), and the norm behind it, its gate, the residual and the norm
before the next block are one pass (block_norm).  The fields, and the Fourier layer that reads a frame, are those of fields_in_time.py.

Training clips the gradients of all weights by their norm (clip_grad_norm); the rollout keeps a state of `width` numbers a block and goes on token by token
(gated_recurrence_step).  The maps and the optimiser are PyTorch's, the rest is the library's.

    python examples/blocks_in_time.py --steps 200
"""
import argparse
import os
import sys

import torch
import torch.nn.functional as F

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
from fields_in_time import fields, loss_of  # noqa: E402
from paper_2504_11681_amd import binding as tfno  # noqa: E402


def like(t, dtype=None):
    return None if t is None else torch.empty(t.shape, dtype=dtype or t.dtype, device=t.device)


class GatedRecurrence(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, gate, input_gate, rate):
        """Outputs and the state after the last token."""
        y, final = like(x), torch.empty(x.shape[0], x.shape[2], device=x.device)
        tape = tfno.gated_recurrence_tape(x) if any(ctx.needs_input_grad) else None
        tfno.gated_recurrence(x, gate, input_gate, rate, y, normalise=True, final_state=final, tape=tape)
        if tape is not None:
            ctx.save_for_backward(x, gate, input_gate, rate, tape)
        return y, final

    @staticmethod
    def backward(ctx, d_y, d_final):
        *inputs, tape = ctx.saved_tensors
        d = [like(t) for t in inputs]
        tfno.gated_recurrence_backward(*inputs, d_y.contiguous(), *d, tape, normalise=True, d_final_state=d_final.contiguous())
        return tuple(d)


class BlockNorm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, y, r, gate, w_after, w_before):
        """The residual stream behind a block, and what the next block reads."""
        ctx.save_for_backward(y, r, gate, w_after, w_before)
        return tfno.block_norm(y, r, gate, w_after, w_before, like(r), like(y))

    @staticmethod
    def backward(ctx, d_r, d_n):
        inputs = ctx.saved_tensors
        d = [like(t) for t in inputs]
        tfno.block_norm_backward(*inputs, d_r.contiguous(), d_n.contiguous(), *d)
        return tuple(d)


class BlocksInTime(torch.nn.Module):
    """u[B, T, N] to the next frames; `dtype` is what the blocks are held in, the residual stream is float32."""

    def __init__(self, N=256, modes=24, channels=4, points=32, width=128, blocks=2, dtype=torch.bfloat16):
        super().__init__()
        self.N, self.channels, self.points, self.dtype = N, channels, points, dtype
        seen = channels * points
        self.enter = torch.nn.Linear(seen, width)
        self.maps = torch.nn.ModuleList(torch.nn.Linear(width, 3 * width) for _ in range(blocks))
        # states that last from two tokens to some hundred
        self.rate = torch.nn.Parameter(torch.linspace(-5.0, 0.5, width).repeat(blocks, 1))
        self.gate = torch.nn.Parameter(torch.full((blocks, width), 0.5))
        self.w_after, self.w_before = (torch.nn.Parameter(torch.ones(blocks, width)) for _ in range(2))
        self.next = torch.nn.Linear(width, N)
        with torch.no_grad():                              # the change of a frame starts at zero
            self.next.weight.mul_(0.1), self.next.bias.zero_()
        self.register_buffer("modes", torch.randn(1, channels, modes, dtype=torch.complex64))     # features of a frame; not trained

    def see(self, u):
        """u[B, T, N] to the residual stream, and what the first block reads."""
        B, T, N = u.shape
        y = torch.empty(B * T, self.channels, N, device=u.device)
        tfno.fno1d_real(u.reshape(B * T, 1, N).contiguous(), self.modes, y)
        r = self.enter(y[:, :, ::N // self.points].reshape(B, T, -1))
        return r, r.to(self.dtype)

    def into(self, i, n):
        """What block i mixes along time, its two gates, and the rates of its channels."""
        x, gate, input_gate = self.maps[i](n.float()).to(self.dtype).chunk(3, -1)
        return x, gate, input_gate, F.softplus(self.rate[i])

    def forward(self, u):
        """The frames after u[B, T, N], and the states that a rollout goes on from."""
        r, n = self.see(u)
        states = []
        for i in range(len(self.maps)):
            y, state = GatedRecurrence.apply(*self.into(i, n))
            states.append(state)
            r, n = BlockNorm.apply(y, r, self.gate[i], self.w_after[i], self.w_before[i])
        return u + self.next(n.float()), states

    @torch.no_grad()
    def step(self, u, states):
        """The frame after u[B, N]; advances the states."""
        r, n = self.see(u[:, None])
        for i, state in enumerate(states):
            x, gate, input_gate, rate = self.into(i, n[:, 0])
            y = torch.empty(x.shape, dtype=x.dtype, device=x.device)
            tfno.gated_recurrence_step(x, gate, input_gate, rate, state, y, normalise=True)
            r, n = tfno.block_norm(y[:, None], r, self.gate[i], self.w_after[i], self.w_before[i], like(r), like(n))
        return u + self.next(n[:, 0].float())


def train(model, steps, B=16, T=129, lr=2e-3, limit=1.0, seed=1, say=print):
    gen = torch.Generator("cuda").manual_seed(seed)
    optimizer = torch.optim.Adam(model.parameters(), lr=lr)
    norm, losses = torch.empty((), device="cuda"), []
    for i in range(steps):
        optimizer.zero_grad()
        loss = loss_of(model, fields(B, T, model.N, gen))
        loss.backward()
        tfno.clip_grad_norm([p.grad for p in model.parameters()], limit, norm)
        optimizer.step()
        losses.append(float(loss.detach()))
        if i % 20 == 0 or i + 1 == steps:
            say(f"step {i}: error of the next frame {losses[-1]:.4f} of that of the frame before, norm of the gradients {float(norm):.3f}", flush=True)
    return losses


@torch.no_grad()
def rollout(model, u, more):
    """`more` frames after u[B, T, N], each from the one before."""
    predicted, states = model(u)
    frames = [predicted[:, -1]]
    while len(frames) < more:
        frames.append(model.step(frames[-1], states))
    return torch.stack(frames, 1)


def main():
    parser = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    parser.add_argument("--steps", type=int, default=200)
    parser.add_argument("--more", type=int, default=16, help="frames of the rollout")
    a = parser.parse_args()
    torch.manual_seed(0)
    model = BlocksInTime().cuda()
    train(model, a.steps)
    u = fields(8, 128 + a.more, model.N, torch.Generator("cuda").manual_seed(2))
    frames, truth = rollout(model, u[:, :128], a.more), u[:, 128:]
    for n in sorted({1, a.more // 2, a.more} - {0}):
        still = (u[:, 127] - truth[:, n - 1]).norm() / truth[:, n - 1].norm()
        print(f"{n} frames on: off by {float((frames[:, n - 1] - truth[:, n - 1]).norm() / truth[:, n - 1].norm()):.3f}, the last frame seen by {float(still):.3f}")


if __name__ == "__main__":
    main()
