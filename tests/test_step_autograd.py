"""What autograd sees of the local step's operators.  The kernels' calls are replaced by plain stand-ins on the host."""
from __future__ import annotations

import pytest
import torch

from paper_2506_04531_b200 import step


@pytest.fixture
def plain(monkeypatch):
    """Stand-ins with the calls' signatures: a rotation by 90 degrees, uniform attention, and a quadratic loss."""
    def rope(q, k, freqs, *, inverse=False, **how):
        sign = -1.0 if inverse else 1.0
        turned = lambda x: None if x is None else torch.cat([-sign * x[..., 1:2], sign * x[..., :1], x[..., 2:]], -1)  # noqa: E731
        return turned(q.detach()), turned(None if k is None else k.detach())

    def attention_forward(q, k, v, **how):
        return v.detach().mean(1, keepdim=True).expand_as(q).contiguous(), q.new_zeros(q.shape[0], q.shape[2], q.shape[1])

    def attention_backward(dout, q, k, v, o, lse, **how):
        return torch.zeros_like(q), torch.zeros_like(k), dout.mean(1, keepdim=True).expand_as(v).contiguous()

    def distill_forward(z, *rest, **how):
        return z.detach().pow(2).sum(1) / 2, z.new_zeros(z.shape[0], 2)

    def distill_backward(dloss, z, *rest, **how):
        return z.detach() * dloss[:, None]

    for f in (rope, attention_forward, attention_backward, distill_forward, distill_backward):
        monkeypatch.setattr(step, f.__name__, f)


def test_rotary_without_keys_has_a_gradient(plain):
    q = torch.randn(1, 3, 2, 8, requires_grad=True)
    w = torch.randn(1, 3, 2, 8)
    y, none = step.rotary(q, None, torch.ones(1, dtype=torch.float64))
    assert none is None
    (y * w).sum().backward()
    assert torch.equal(q.grad, step.rope(w, None, None, inverse=True)[0])


def test_rotary_where_only_the_keys_are_used(plain):
    q, k = torch.randn(1, 3, 2, 8, requires_grad=True), torch.randn(1, 3, 2, 8, requires_grad=True)
    step.rotary(q, k, torch.ones(1, dtype=torch.float64))[1].sum().backward()
    assert float(q.grad.abs().sum()) == 0 and torch.equal(k.grad, step.rope(torch.ones_like(k), None, None, inverse=True)[0])


def test_rotary_twice_differentiated(plain):
    """Linear in q: the penalty on a gradient sees the way there and back."""
    q, w = torch.randn(1, 3, 2, 8, requires_grad=True), torch.randn(1, 3, 2, 8)
    y = step.rotary(q, None, torch.ones(1, dtype=torch.float64))[0]
    g, = torch.autograd.grad((y.pow(3) * w).sum(), q, create_graph=True)
    second, = torch.autograd.grad(g.sum(), q)
    turn = lambda x, inverse=False: step.rope(x, None, None, inverse=inverse)[0]  # noqa: E731
    want = turn(6 * turn(q) * w * turn(torch.ones_like(q)), True)
    assert torch.allclose(second, want, atol=1e-5)


@pytest.mark.parametrize("last", [True, False])
def test_a_second_derivative_of_attention_is_refused_and_not_left_out(plain, last):
    """Where attention comes last, the gradient of its output is a constant: the term that would be dropped is that of q, k and v."""
    q, k, v = (torch.randn(1, 3, 2, 8, requires_grad=True) for _ in range(3))
    o = step.attention(q, k, v)
    grads = torch.autograd.grad(o.sum() if last else o.pow(2).sum(), (q, k, v), create_graph=True)
    penalty = sum(g.pow(2).sum() for g in grads) + v.pow(2).sum()
    with pytest.raises(step.HalosError, match="second derivative"):
        penalty.backward()


@pytest.mark.parametrize("last", [True, False])
def test_a_second_derivative_of_the_loss_is_refused_and_not_left_out(plain, last):
    z = torch.randn(3, 5, requires_grad=True)
    loss = step.distill_loss(z, None)
    g, = torch.autograd.grad(loss.sum() if last else loss.pow(2).sum(), z, create_graph=True)
    with pytest.raises(step.HalosError, match="second derivative"):
        (g.pow(2).sum() + z.sum()).backward()


def test_first_derivatives_with_a_graph_are_the_same(plain):
    z = torch.randn(3, 5, requires_grad=True)
    a, = torch.autograd.grad(step.distill_loss(z, None).sum(), z)
    b, = torch.autograd.grad(step.distill_loss(z, None).sum(), z, create_graph=True)
    assert torch.equal(a, b)
    v = torch.randn(1, 3, 2, 8, requires_grad=True)
    a, = torch.autograd.grad(step.attention(v.detach(), v.detach(), v).pow(2).sum(), v)
    b, = torch.autograd.grad(step.attention(v.detach(), v.detach(), v).pow(2).sum(), v, create_graph=True)
    assert torch.equal(a, b)


@pytest.mark.parametrize("what", ["doc_start", "lens"])
def test_a_mask_that_is_overwritten_before_the_backward_pass_is_noticed(plain, what):
    """A buffer that the next batch's documents are written to."""
    v = torch.randn(2, 3, 2, 8, requires_grad=True)
    mask = torch.zeros((2, 3) if what == "doc_start" else (2,), dtype=torch.int32)
    step.attention(v.detach(), v.detach(), v, **{what: mask}).sum().backward()
    o = step.attention(v.detach(), v.detach(), v, **{what: mask})
    mask += 1
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        o.sum().backward()
