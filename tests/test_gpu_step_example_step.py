"""The example's local step against the same step written plainly from the same gradient, and its schedule."""
from __future__ import annotations

import pytest
import torch

import step_more_oracle as mo
from paper_2506_04531_b200 import step
from paper_2506_04531_b200.examples import local_steps as ex
from paper_2506_04531_b200.inputs import gen, layouts

pytestmark = pytest.mark.gpu
RATE = 0.25


def _start(norm):
    layout = layouts.decoder_layout("example", ex.LAYERS, ex.WIDTH, ex.VOCAB)
    flat = torch.from_numpy(gen.theta_init(layout, 0)).cuda()
    flat += 0.02 * torch.randn(flat.shape, generator=torch.Generator(device="cuda").manual_seed(1), device="cuda")
    return ex.Decoder(layout, norm), flat, ex.documents(torch.Generator().manual_seed(2))


def _gradient(model, flat, batch):
    tokens, labels, positions, starts = batch
    a = flat.clone().requires_grad_()
    loss = step.distill_loss(model.logits(a, tokens, positions, starts), labels.reshape(-1), mix=0.0, temperature=2.0)
    return torch.autograd.grad(loss.sum() / (labels != -100).sum(), a)[0]


@pytest.mark.parametrize("norm", ["layer", "rms"])
@pytest.mark.parametrize("part", [0.25, 4.0, None])
def test_one_step(norm, part):
    """max_norm at a quarter of the gradient's norm, above it, and none: the step is that of the formula, its direction, rate and factor."""
    model, flat, batch = _start(norm)
    grad = _gradient(model, flat, batch)
    length = mo.norm([grad])
    limit = None if part is None else float(torch.tensor(part * length, dtype=torch.float32))
    theta, _ = ex.local_steps(model, flat, None, [batch], RATE, 0.0, limit)
    factor = 1.0 if limit is None else min(1.0, limit / length)
    moved = RATE * factor * grad.double()
    want = flat.double() - moved
    # the factor is off by the norm's error and its own rounding, the product and the difference are rounded once each
    mo.close(theta, want, mo.rounded(want, 9 * mo.E * moved.abs() + mo.E * want.abs(), torch.float32))
    assert float(moved.abs().max()) > 1000 * mo.E * float(flat.abs().max())      # the step can be told from none


def test_the_schedule():
    """Ten results of four workers in turn, two of them under each server: a server pushes with every fourth that it gets."""
    losses, counters = ex.run(rounds=10, h_steps=1, norm="rms", max_norm=0.5, log=None)
    assert len(losses) == 10 and counters["t"] == 6 and counters["i"] == 2
    assert not step.fault()
