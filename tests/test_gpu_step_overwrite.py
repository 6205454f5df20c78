"""Tensors that the local step's operators write over, as autograd sees them."""
from __future__ import annotations

import pytest
import torch

from paper_2506_04531_b200 import binding as hb, step

pytestmark = pytest.mark.gpu


def _rope(x):
    return step.rope(x, None, step.rotary_frequencies(8)[0], inplace=True)


def _loss(x):
    z = x.view(4, 64)
    ones = torch.ones(4, device="cuda")
    return step.distill_loss_and_grad(z.detach().clone(), torch.zeros(4, dtype=torch.int64, device="cuda"), None, None, ones, out=z)


def _loss_backward(x):
    z = x.view(4, 64)
    return step.distill_backward(torch.ones(4, device="cuda"), z, torch.zeros(4, 2, device="cuda"), torch.zeros(4, dtype=torch.int64, device="cuda"), None, None, out=z)


@pytest.mark.parametrize("write", [_rope, _loss, _loss_backward])
def test_a_saved_tensor_that_is_overwritten_is_noticed(write):
    w = torch.randn(1, 4, 4, 16, device="cuda", requires_grad=True)
    x = torch.randn(1, 4, 4, 16, device="cuda")
    y = (w * x).sum()                       # saves x
    write(x)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.backward()


@pytest.mark.parametrize("write", [_rope, _loss, _loss_backward])
def test_a_tensor_in_a_graph_is_not_overwritten(write):
    w = torch.randn(1, 4, 4, 16, device="cuda", requires_grad=True)
    x = w * 2
    before = x.detach().clone()
    with pytest.raises(hb.HalosError) as e:
        write(x)
    assert e.value.status == hb.ERR_INVALID_ARG and torch.equal(x, before)
    with torch.no_grad():
        write(x)
    write(x.detach())
    with torch.inference_mode():
        write(torch.randn(1, 4, 4, 16, device="cuda"))
