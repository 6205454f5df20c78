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


@pytest.mark.parametrize("residual", [False, True])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("d,loose", [(8, False), (250, True), (1021, False), (2048, False), (9000, False), (40000, False)])
def test_rows_of_subnormal_elements(d, loose, dtype, residual):
    """One over their root mean square is more than 32 bits hold; the normalised row is not."""
    least = 2.0 ** (-149 if dtype == F32 else -133)
    k = torch.randint(-15, 16, (5, d), generator=torch.Generator(device="cuda").manual_seed(4), device="cuda")
    k[:, 0] = 7
    k[3] *= 1 << 20                                     # a row that 32 bits do hold
    x = (k.double() * least).to(dtype)
    if loose:
        x = torch.cat([x, x[:, :1]], 1)[:, :d]
    r = x.contiguous() if residual else None
    w = _x((d,), F32, 5)
    y, summed, rstd = step.rms_norm_forward(x, w, residual=r, eps=0.0)
    o = mo.rms_norm(x, w, r, 0.0)
    mo.close(y, o["y"], mo.rounded(o["y"], o["y_off"], dtype))
    held = o["rstd"] < 3.4e38
    assert int(held.sum()) == 1 and bool(rstd[~held].isinf().all())
    mo.close(rstd[held], o["rstd"][held], o["rstd_bound"][held])
    for group in (0, 64):
        q, scales, _, again = step.rms_norm_quantized(x, w, residual=r, eps=0.0, group=group)
        assert torch.equal(again, rstd)
        wide = torch.repeat_interleave(scales.double(), group or d, -1)[..., :d]
        # half a step of what is held: 2^-4 of a normal value, 2^-10 below 2^-6; the quotient is rounded once before, and the scale once
        mo.close(q.double() * wide, o["y"], torch.maximum(2.0 ** -4 * (o["y"].abs() + o["y_off"]) * (1 + 4 * mo.E), 2.0 ** -10 * wide) + o["y_off"] + 4 * mo.E * o["y"].abs())


@pytest.mark.parametrize("dtype,wtype", [(F32, F32), (BF16, F32), (F16, F16)])
@pytest.mark.parametrize("d", [508, 510, 516, 765, 766, 772, 3076, 4093, 4094, 4100, 6141, 6142, 6144, 6148, 8190, 8196, 12287, 12289, 12296, 16376, 16377, 16378, 16384, 16385, 16392])
def test_on_both_sides_of_where_other_kernels_take_over(d, dtype, wtype):
    """Rows that a CTA holds in one way or another, and rows that go through loops; on 16 bytes as they lie in memory of their own, off them, and in strides apart."""
    rows = 19
    for how in ("whole", "apart"):
        x, r, dy, ds = (_x((rows, d), dtype, s) for s in (6, 7, 8, 9))
        if how == "apart":
            x = torch.cat([x, x[:, :1]], 1)[:, :d]
        w = (1 + _x((d,), F32, 10, 0.2)).to(wtype)
        for residual in (None, r):
            got = step.rms_norm_forward(x, w, residual=residual)
            o = mo.rms_norm(x, w, residual, 1e-5)
            mo.close(got[0], o["y"], mo.rounded(o["y"], o["y_off"], dtype))
            mo.close(got[2], o["rstd"], o["rstd_bound"])
            if residual is not None:
                mo.close(got[1], o["summed"], o["summed_bound"])
            for group in (0, 64):
                q, scales, _, rstd = step.rms_norm_quantized(x, w, residual=residual, group=group)
                want, want_scales = _in_8_bits(x, residual, w, rstd, group)
                assert torch.equal(scales, want_scales) and torch.equal(q.view(torch.uint8), want)
            for dsummed in (None, ds):
                dx, dw = step.rms_norm_backward(dy, got[1], w, got[2], dsummed=dsummed)
                b = mo.rms_norm_backward(dy, got[1], w, got[2], dsummed)
                mo.close(dx, b["dx"], b["dx_bound"])
                mo.close(dw, b["dw"], b["dw_bound"])
