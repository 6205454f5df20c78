"""CPU-side checks at the limits of the embedding's, the norms' and the gradients' calls, with stand-ins for the kernels."""
from __future__ import annotations

import re
from pathlib import Path

import pytest
import torch

from paper_2506_04531_b200 import step

CSRC = Path(step.__file__).resolve().parent / "csrc"


@pytest.fixture
def plain(monkeypatch):
    """The embedding as the interface has it: a token outside the vocabulary gives a row of NaN and takes no part in the gradient."""
    def embedding_forward(weight, tokens, *, scale=1.0, dtype=None):
        known = (tokens >= 0) & (tokens < weight.size(0))
        rows = weight.detach()[tokens.clamp(0, weight.size(0) - 1)] * scale
        return torch.where(known[..., None], rows, float("nan")).to(dtype or weight.dtype)

    def embedding_backward(dout, tokens, vocab, *, scale=1.0, dtype=None, **kw):
        flat, rows = tokens.reshape(-1), dout.detach().reshape(-1, dout.size(-1))
        known = (flat >= 0) & (flat < vocab)
        return (dout.new_zeros(vocab, dout.size(-1)).index_add(0, flat[known], rows[known]) * scale).to(dtype or dout.dtype)

    for f in (embedding_forward, embedding_backward):
        monkeypatch.setattr(step, f.__name__, f)


def test_second_derivatives_leave_out_tokens_that_are_none(plain):
    w, t = torch.randn(6, 4, dtype=torch.float64, requires_grad=True), torch.tensor([[1, -1, 5], [6, 1, -100]])
    known = (t >= 0) & (t < 6)
    dout = torch.randn(2, 3, 4, dtype=torch.float64, requires_grad=True)
    y = step.embedding(w, t, scale=2.0)
    g, = torch.autograd.grad(y, w, dout, create_graph=True)
    first, = torch.autograd.grad(g.pow(3).sum(), dout, create_graph=True)
    with torch.no_grad():
        want = torch.where(known[..., None], 2.0 * 3 * g.pow(2)[t.clamp(0, 5)], 0.0)
    assert torch.equal(first, want)
    again, = torch.autograd.grad(first.sum(), dout)     # and once more: 24 g of each row, for every place of its token
    counts = torch.bincount(t[known], minlength=6).double()
    with torch.no_grad():
        want = torch.where(known[..., None], (24.0 * g * counts[:, None])[t.clamp(0, 5)], 0.0)
    assert torch.allclose(again, want)


@pytest.mark.parametrize("kernel,names", [("embedding_sort_kernel", ["s_count"]), ("embedding_sum_kernel", ["s_head", "s_tail"])])
def test_shared_arrays_with_accesses_of_16_bytes_are_aligned_to_them(kernel, names):
    """Their types alone ask for 2 or 4 bytes, and smaller variables lie beside them."""
    body = (CSRC / "step_embedding.cu").read_text().split(kernel + "(", 1)[1].split("\n}\n", 1)[0]
    for name in names:
        line, = re.findall(rf"^ *(__shared__ [^;]*\b{name}\[[^;]*);", body, re.M)
        assert line.startswith("__shared__ __align__(16) "), line


def test_matrices_that_share_memory():
    """Against sets of bytes: rows of any distance, one row, rows that overlap one another or are all the same, and rows of one between those of the other."""
    import random
    rng, seen = random.Random(0), {False: 0, True: 0}
    for _ in range(4000):
        a, b = ((rng.randrange(60), rng.randrange(5), rng.choice([0, 3, 8, 12, 16, 24]), rng.randrange(9)) for _ in range(2))
        bytes_of = lambda m: {m[0] + i * m[2] + k for i in range(m[1]) for k in range(m[3])}  # noqa: E731
        want = bool(bytes_of(a) & bytes_of(b))
        assert step._share(a, b) is want and step._share(b, a) is want, (a, b)
        seen[want] += 1
    assert min(seen.values()) > 500


def test_shared_memory_is_looked_for_on_the_host():
    """Whatever device new tensors go to by default: a device's would have to be waited for, which a captured stream cannot be."""
    try:
        torch.set_default_device("meta")
        assert step._share((0, 3, 8, 4), (4, 3, 8, 4)) is False and step._share((0, 3, 8, 4), (3, 3, 8, 4)) is True
    finally:
        torch.set_default_device(None)
