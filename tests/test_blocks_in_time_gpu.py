"""The example that trains and rolls out blocks of the gated recurrence: it runs, its gradient is that of its loss, and token by token it gives what it gives over whole
sequences."""
import math
import os
import sys

import pytest
import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def example():
    import blocks_in_time
    assert torch.cuda.is_available(), "these tests need the MI355X"
    blocks_in_time.tfno.lib()
    return blocks_in_time


def test_runs(example):
    torch.manual_seed(0)
    model = example.BlocksInTime(points=16, width=48).cuda()
    before = [p.detach().clone() for p in model.parameters()]
    losses = example.train(model, 3, B=4, T=40)
    assert all(math.isfinite(v) for v in losses)
    assert all(torch.isfinite(p).all() for p in model.parameters())
    assert sum(not torch.equal(p, b) for p, b in zip(model.parameters(), before)) == len(before)
    u = example.fields(2, 40, model.N, torch.Generator("cuda").manual_seed(2))
    assert torch.isfinite(example.rollout(model, u, 4)).all()


def test_gradient_against_differences(example):
    """Along the gradient itself: central differences at two steps, joined so that what is left of third order in the step cancels.  The loss is some thousand float32 terms,
    1e-6 off at most; over a change of 2e-3 or more that is 1e-3."""
    torch.manual_seed(0)
    model = example.BlocksInTime(points=8, width=24, dtype=torch.float32).cuda()
    u = example.fields(3, 80, model.N, torch.Generator("cuda").manual_seed(3))
    loss = example.loss_of(model, u)
    loss.backward()
    weights = list(model.parameters())
    grads = [w.grad.clone() for w in weights]
    norm = torch.sqrt(sum(g.double().square().sum() for g in grads))
    start = [w.detach().clone() for w in weights]

    @torch.no_grad()
    def at(step):
        for w, s, g in zip(weights, start, grads):
            w.copy_(s + step * g / norm)
        return float(example.loss_of(model, u).double())

    h = 2e-3 * float(loss.detach()) / float(norm)          # the loss changes by some 2e-3 of itself to either side
    slopes = [(at(s) - at(-s)) / (2 * s) for s in (h, h / 2)]
    slope = (4 * slopes[1] - slopes[0]) / 3
    print("slope", slope, "norm of the gradient", float(norm), flush=True)
    assert abs(slope - float(norm)) <= 1e-2 * float(norm)
    limited = [g.clone() for g in grads]
    kept = torch.empty((), device="cuda")
    example.tfno.clip_grad_norm(limited, 0.5 * float(norm), kept)
    assert abs(float(kept) - float(norm)) <= 2.0 ** -22 * float(norm)
    assert all(((a - 0.5 * b).abs() <= 2.0 ** -22 * b.abs()).all() for a, b in zip(limited, grads))


@pytest.mark.parametrize("dtype, bound", ((torch.float32, 2.0 ** -16), (torch.bfloat16, 2.0 ** -6)))
def test_steps_follow_the_whole_sequence(example, dtype, bound):
    """The change of a frame is a sum over values that were rounded once each in every block: inputs, gates and outputs in BF16, 2^-8 each; in float32 states and products of
    some hundred terms, 2^-24 each."""
    torch.manual_seed(0)
    model = example.BlocksInTime(points=16, width=48, dtype=dtype).cuda()
    u = example.fields(4, 70, model.N, torch.Generator("cuda").manual_seed(4))
    with torch.no_grad():
        whole, final = model(u)
        states = [torch.zeros_like(s) for s in final]
        steps = torch.stack([model.step(u[:, t], states) for t in range(u.shape[1])], 1)
    off = float(((steps - u) - (whole - u)).norm() / (whole - u).norm())
    print("frames", off, "states", [float((a - b).norm() / b.norm()) for a, b in zip(states, final)], flush=True)
    assert off <= bound
    assert all(float((a - b).norm() / b.norm()) <= bound for a, b in zip(states, final))
