"""The embedding at the limits of its interface: derivatives of the gradient for tokens that are none, and what may lie in one run of memory."""
from __future__ import annotations

import pytest
import torch

from paper_2506_04531_b200 import step

pytestmark = pytest.mark.gpu


def _x(shape, seed, dtype=torch.float32):
    return torch.randn(shape, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda").to(dtype)


@pytest.mark.parametrize("kind", [torch.int32, torch.int64])
def test_second_derivatives_leave_out_tokens_that_are_none(kind):
    """Of the gradient's square, with padding among the tokens: powers of two throughout, so that nothing is rounded."""
    t = torch.tensor([[1, -1, 5, 5], [20, 1, -100, 3]], dtype=kind, device="cuda")
    known = ((t >= 0) & (t < 20))[..., None]
    w = torch.ones((20, 16), device="cuda", requires_grad=True)
    dout = torch.full((2, 4, 16), 0.5, device="cuda", requires_grad=True)
    g, = torch.autograd.grad(step.embedding(w, t, scale=4.0), w, dout, create_graph=True)
    got, = torch.autograd.grad(g.pow(2).sum(), dout)
    with torch.no_grad():
        assert torch.equal(got, torch.where(known, 8.0 * g[t.long().clamp(0, 19)], 0.0))
