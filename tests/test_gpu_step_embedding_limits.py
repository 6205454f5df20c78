"""The embedding at the limits of its interface: derivatives of the gradient for tokens that are none, and what may lie in one run of memory."""
from __future__ import annotations

import pytest
import torch

from paper_2506_04531_b200 import binding as hb, step

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


@pytest.mark.parametrize("accumulate", [False, True])
def test_a_gradient_is_not_written_over_what_it_is_formed_from(accumulate):
    t = torch.randint(0, 50, (40,), generator=torch.Generator(device="cuda").manual_seed(1), device="cuda")
    room = _x((50, 64), 2)
    kw = dict(accumulate=accumulate)
    for dout, out, tokens in ((room[:40], room, t), (room[10:], room, t), (room[:40, :32], room[:, 31:63], t), (room[:1].expand(40, -1), room, t), (room.view(-1)[5:5 + 40 * 64].view(40, 64), room, t),
                              (_x((40, 64), 3), room, room.view(torch.int64).view(-1)[100:140]), (room.bfloat16()[:40, :32], room.view(torch.bfloat16)[:, :32], room.view(torch.int32)[3, :40])):
        before = room.clone()
        with pytest.raises(hb.HalosError, match="shares memory") as e:
            step.embedding_backward(dout, tokens, 50, out=out, **kw)
        assert e.value.status == hb.ERR_INVALID_ARG and torch.equal(room, before)
    # side by side in one run of memory, and one behind the other
    both = _x((50, 128), 4)
    want = step.embedding_backward(both[:40, :64].clone(), t, 50, out=both[:, 64:].clone(), **kw)
    assert torch.equal(step.embedding_backward(both[:40, :64], t, 50, out=both[:, 64:], **kw), want)
    want = step.embedding_backward(room[:40].clone(), t, 50, out=_x((50, 64), 5), **kw)
    stack = torch.cat([room[:40], _x((50, 64), 5)])
    assert torch.equal(step.embedding_backward(stack[:40], t, 50, out=stack[40:], **kw), want)
