"""The example that runs the Fourier layer, the norm with rotation and the gated delta rule together: it learns, its gradient is that of its loss, and
token by token it gives what it gives over whole sequences."""
import os
import sys

import pytest
import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def example():
    import fields_in_time
    assert torch.cuda.is_available(), "these tests need the MI355X"
    fields_in_time.tfno.lib()
    return fields_in_time


def test_learns(example):
    torch.manual_seed(0)
    losses = example.train(example.FieldsInTime(points=16, D=32).cuda(), 80, B=8, T=70)
    assert sum(losses[-5:]) < 0.5 * sum(losses[:5]), losses


def test_gradient_against_differences(example):
    """Along the gradient itself, where the loss changes fastest: central differences at two steps, joined so that what is left of third order in the step
    cancels.  The loss is some thousand float32 terms, 1e-6 off at most; over a change of 2e-3 or more that is 1e-3."""
    torch.manual_seed(0)
    model = example.FieldsInTime(points=8, D=16, dtype=torch.float32).cuda()
    u = example.fields(3, 80, model.N, torch.Generator("cuda").manual_seed(3))
    with torch.no_grad():
        model.skip.weight.normal_(std=0.02)
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


@pytest.mark.parametrize("dtype, bound", ((torch.float32, 2.0 ** -16), (torch.bfloat16, 2.0 ** -6)))
def test_steps_follow_the_whole_sequence(example, dtype, bound):
    """The change of a frame is a sum over values that were rounded once each: queries, keys, values and outputs in BF16, 2^-8 each."""
    torch.manual_seed(0)
    model = example.FieldsInTime(points=16, D=32, dtype=dtype).cuda()
    u = example.fields(4, 70, model.N, torch.Generator("cuda").manual_seed(4))
    with torch.no_grad():
        whole, final = model(u)
        state = torch.zeros_like(final)
        steps = torch.stack([model.step(u[:, t], t, state) for t in range(u.shape[1])], 1)
    off = float(((steps - u) - (whole - u)).norm() / (whole - u).norm())
    states = float((state - final).norm() / final.norm())
    print("frames", off, "states", states, flush=True)
    assert off <= bound and states <= bound


def test_rollout_goes_on_from_the_state(example):
    torch.manual_seed(0)
    model = example.FieldsInTime(points=16, D=32, dtype=torch.float32).cuda()
    u = example.fields(4, 70, model.N, torch.Generator("cuda").manual_seed(5))
    frames = example.rollout(model, u, 3)
    for n in range(3):                                     # the same frames from whole sequences
        with torch.no_grad():
            again = model(torch.cat([u, frames[:, :n]], 1))[0][:, -1]
        off = float((frames[:, n] - again).norm() / again.norm())
        print(n, off, flush=True)
        assert off <= 2.0 ** -16
