"""Root-mean-square norms where single roundings and the range of 32 bits show: 8-bit values next to the middle of two, rows of subnormal elements."""
from __future__ import annotations

import pytest
import torch

import step_more_oracle as mo
from paper_2506_04531_b200 import step

pytestmark = pytest.mark.gpu
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16


def _x(shape, dtype, seed, scale=1.0):
    return (torch.randn(shape, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda") * scale).to(dtype)


def _in_8_bits(x, residual, weight, rstd, group):
    """(bytes, scales) by the interface's formula, an operation at a time: every one of these is correctly rounded in 32 bits."""
    s = x.float() if residual is None else x.float() + residual.float()
    y = s * rstd[..., None] * weight.float()
    d = y.shape[-1]
    n = group or d
    pieces = torch.cat([y, y.new_zeros((*y.shape[:-1], -d % n))], -1).unflatten(-1, (-1, n))
    scales = (pieces.abs().amax(-1) * torch.tensor(1 / 448, dtype=F32, device=y.device)).clamp_min(2.0 ** -126)
    return (pieces / scales[..., None]).flatten(-2)[..., :d].to(torch.float8_e4m3fn).view(torch.uint8), scales


@pytest.mark.parametrize("group", [0, 32, 64, 128])
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("d,loose", [(56, False), (80, False), (250, True), (1021, False), (2048, False), (4100, False), (7168, False), (40000, False)])
def test_8_bits_are_the_nearest_to_the_quotient(d, loose, dtype, group):
    """Bit for bit, wherever rows begin and however they are held.  Elements and weights of few bits meet the middle between two 8-bit values often: some of 10^5 quotients
    lie within 2^-23 of one."""
    rows = (1 << 21) // d
    x, r = _x((rows, d), dtype, 1, 1.5).bfloat16().to(dtype), _x((rows, d), dtype, 2, 1.5).bfloat16().to(dtype)
    w = (1 + _x((d,), F32, 3, 0.1)).bfloat16()
    if loose:
        x = torch.cat([x, x[:, :1]], 1)[:, :d]          # rows of x and r begin differently far behind 16 bytes
    x[0] = 0
    for residual in (None, r):
        q, scales, _, rstd = step.rms_norm_quantized(x, w, residual=residual, group=group)
        want, want_scales = _in_8_bits(x, residual, w, rstd, group)
        assert torch.equal(scales, want_scales)
        assert int((q.view(torch.uint8) != want).sum()) == 0
