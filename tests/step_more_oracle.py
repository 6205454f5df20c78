"""Plain 64-bit forms of the embedding, the norms and what happens to gradients, and the error bounds that follow from where the kernels round.

Nothing here comes from the CUDA library.  E is half the spacing of 32-bit floats at 1: one product, or one sum, is off by at most E of itself."""
from __future__ import annotations

import torch

from step_oracle import TINY, U

E = 2.0 ** -24


def rounded(want, off, dtype):
    """The bound of a value that is off by `off` before it is rounded to dtype."""
    return off if dtype == torch.float64 else off + U[dtype] * (want.abs() + off) + TINY[dtype]


def close(got, want, bound):
    """NaN and infinities in the same places, the rest within the bound."""
    got, want = got.double(), want.double()
    assert got.shape == want.shape
    fine = torch.isfinite(want)
    assert torch.equal(torch.isnan(got), torch.isnan(want)), "NaN in other places"
    assert torch.equal(got[~fine].nan_to_num(0.0), want[~fine].nan_to_num(0.0)), "other infinities"
    off = (got - want).abs()[fine] - bound.expand_as(want)[fine]
    assert off.numel() == 0 or float(off.max()) <= 0, float(off.max())


def embedding(weight, tokens, scale, dtype):
    """(rows, bound); a token outside the vocabulary gives NaN."""
    t = tokens.long()
    known = (t >= 0) & (t < weight.shape[0])
    want = scale * weight.double()[t.clamp(0, weight.shape[0] - 1)]
    want = torch.where(known[..., None], want, float("nan"))
    return want, rounded(want, E * want.abs(), dtype)


def embedding_backward(dout, tokens, vocab, scale, dtype, before=None):
    """(gradient, bound): a sum of n terms in any order is off by at most n E times the sum of their sizes."""
    t, d = tokens.long().reshape(-1), dout.double().reshape(-1, dout.shape[-1])
    known = (t >= 0) & (t < vocab)
    t, d = t[known], d[known]
    z = torch.zeros((vocab, d.shape[1]), dtype=torch.float64, device=d.device)
    want, size = z.index_add(0, t, d) * scale, z.index_add(0, t, d.abs()) * abs(scale)
    n = torch.bincount(t, minlength=vocab)[:, None].double()
    off = (n + 1) * E * size
    if before is not None:
        want = want + before.double()
        off = off + E * want.abs()
    return want, rounded(want, off, dtype)


def _sum_off(d):
    """Relative, of a sum of d terms of one sign: a thread adds up to 32 of them, or d / 256 where rows are longer, then its warp and the other warps."""
    return (32 + d / 256 + 5 + 32) * E


def rms_norm(x, weight, residual, eps):
    """A dict of y (before it is rounded), its error, summed and rstd with bounds."""
    d = x.shape[-1]
    s = x.double() if residual is None else x.double() + residual.double()
    size = s.abs() if residual is None else x.double().abs() + residual.double().abs()
    mean = (s * s).mean(-1)
    rstd = (mean + eps).rsqrt()
    # s is off by E of x + residual before it is squared; the root halves what the mean is off by; the function itself 2 units of 2^-23
    s_off = torch.zeros_like(size) if residual is None else E * s.abs()
    root_off = rstd * (0.5 * _sum_off(d) + 2 * E + 4 * E + (0 if residual is None else E))
    y = s * rstd[..., None] * weight.double()
    y_off = (s_off * rstd[..., None] + s.abs() * root_off[..., None]) * weight.double().abs() + 2 * E * y.abs()
    return dict(y=y, y_off=y_off, summed=s, summed_bound=rounded(s, s_off, x.dtype), rstd=rstd, rstd_bound=root_off + 1e-38)


def rms_norm_backward(dy, summed, weight, rstd, dsummed):
    d, s, dy64, r = dy.shape[-1], summed.double(), dy.double(), rstd.double()[..., None]
    g, u = dy64 * weight.double(), s * r
    mean, size = (g * u).mean(-1, keepdim=True), (g * u).abs().mean(-1, keepdim=True)
    dx = r * (g - u * mean)
    mean_off = size * (_sum_off(d) + 4 * E)
    dx_off = r * (3 * E * g.abs() + u.abs() * mean_off + 4 * E * (u * mean).abs())
    if dsummed is not None:
        dx = dx + dsummed.double()
        dx_off = dx_off + E * dx.abs()
    rows = max(1, dy.numel() // d)
    dw, dw_size = (dy64 * u).reshape(-1, d).sum(0), (dy64 * u).abs().reshape(-1, d).sum(0)
    return dict(dx=dx, dx_bound=rounded(dx, dx_off, dy.dtype), dw=dw, dw_bound=rounded(dw, (rows + 3) * E * dw_size, weight.dtype))


def norm(grads):
    return float(sum((g.double() ** 2).sum() for g in grads)) ** 0.5


NORM_OFF = 6 * E  # relative: eight squares in 32 bits, halved by the root, and rounded once
