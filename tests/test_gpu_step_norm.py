"""Root-mean-square norms against 64 bits: types, widths, strides, residuals, 8 bits with scales, rows of every size, and their gradient."""
from __future__ import annotations

import math

import pytest
import torch

import step_more_oracle as mo
from paper_2506_04531_b200 import binding as hb, step

pytestmark = pytest.mark.gpu
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
TYPES = [(F32, F32), (BF16, BF16), (F16, F16), (BF16, F32), (F16, F32), (F32, BF16)]    # rows, weight
WIDTHS = [1, 2, 3, 7, 8, 31, 64, 80, 97, 128, 255, 512, 768, 1000, 1021, 1024, 1026, 2048, 2500, 4095, 4096, 8192, 11111]


def _x(shape, dtype, seed, scale=1.0):
    return (torch.randn(shape, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda") * scale).to(dtype)


def _w(d, dtype, seed=99):
    return (1 + 0.2 * _x((d,), F32, seed)).to(dtype)


def _check_forward(x, w, residual, eps, got):
    y, summed, rstd = got
    o = mo.rms_norm(x, w, residual, eps)
    mo.close(y, o["y"], mo.rounded(o["y"], o["y_off"], x.dtype))
    mo.close(rstd, o["rstd"], o["rstd_bound"])
    if residual is None:
        assert summed is x
    else:
        mo.close(summed, o["summed"], o["summed_bound"])


def _check_quantized(x, w, residual, eps, group, got):
    q, scales, summed, rstd = got
    o = mo.rms_norm(x, w, residual, eps)
    d = x.shape[-1]
    n = group or d
    assert q.dtype == torch.float8_e4m3fn and scales.shape == (*x.shape[:-1], -(-d // n))
    pieces = [slice(i, min(d, i + n)) for i in range(0, d, n)]
    top = torch.stack([o["y"][..., p].abs().amax(-1) for p in pieces], -1)
    top_off = torch.stack([o["y_off"][..., p].amax(-1) for p in pieces], -1)
    want = (top / 448).clamp_min(2.0 ** -126)
    mo.close(scales, want, top_off / 448 + 2 * mo.E * want)
    wide = torch.repeat_interleave(scales.double(), n, -1)[..., :d]
    # half a step of what is held: 2^-4 of a normal value, 2^-10 below 2^-6; one product with a reciprocal before
    mo.close(q.double() * wide, o["y"], torch.maximum(2.0 ** -4 * (o["y"].abs() + o["y_off"]) * (1 + 4 * mo.E), 2.0 ** -10 * wide) + o["y_off"] + 4 * mo.E * o["y"].abs())
    mo.close(rstd, o["rstd"], o["rstd_bound"])
    if residual is not None:
        mo.close(summed, o["summed"], o["summed_bound"])


def _check_backward(dy, s, w, rstd, dsummed, got):
    o = mo.rms_norm_backward(dy, s, w, rstd, dsummed)
    mo.close(got[0], o["dx"], o["dx_bound"])
    mo.close(got[1], o["dw"], o["dw_bound"])
    assert got[1].dtype == w.dtype


@pytest.mark.parametrize("dtype,wtype", TYPES)
@pytest.mark.parametrize("d", WIDTHS)
def test_against_64_bits(d, dtype, wtype):
    rows = 37 if d < 3000 else 5
    x, r, w = _x((rows, d), dtype, 1), _x((rows, d), dtype, 2, 3.0), _w(d, wtype)
    for residual in (None, r):
        _check_forward(x, w, residual, 1e-5, step.rms_norm_forward(x, w, residual=residual))
        for group in (0, 32, 64, 128):
            _check_quantized(x, w, residual, 1e-6, group, step.rms_norm_quantized(x, w, residual=residual, eps=1e-6, group=group))
    y, s, rstd = step.rms_norm_forward(x, w, residual=r)
    dy = _x((rows, d), dtype, 3)
    for dsummed in (None, _x((rows, d), dtype, 4)):
        got = step.rms_norm_backward(dy, s, w, rstd, dsummed=dsummed)
        _check_backward(dy, s, w, rstd, dsummed, got)
        assert all(torch.equal(a, b) for a, b in zip(got, step.rms_norm_backward(dy, s, w, rstd, dsummed=dsummed)))


@pytest.mark.parametrize("d", [40000, 70001])
def test_long_rows(d):
    x, r, w = _x((2, 2, d), BF16, 5), _x((2, 2, d), BF16, 6), _w(d, F32)
    got = step.rms_norm_forward(x, w, residual=r)
    _check_forward(x, w, r, 1e-5, got)
    _check_quantized(x, w, r, 1e-5, 128, step.rms_norm_quantized(x, w, residual=r, group=128))
    _check_quantized(x, w, r, 1e-5, 0, step.rms_norm_quantized(x, w, residual=r))
    dy = _x((2, 2, d), BF16, 7)
    _check_backward(dy, got[1], w, got[2], x, step.rms_norm_backward(dy, got[1], w, got[2], dsummed=x))


@pytest.mark.parametrize("rows", [1, 2, 9, 1000, 4099, 30000])
@pytest.mark.parametrize("dtype,d", [(BF16, 256), (F32, 50), (F16, 33)])
def test_numbers_of_rows(rows, dtype, d):
    x, r, w, dy = _x((rows, d), dtype, 8), _x((rows, d), dtype, 9), _w(d, dtype), _x((rows, d), dtype, 10)
    got = step.rms_norm_forward(x, w, residual=r)
    _check_forward(x, w, r, 1e-5, got)
    _check_quantized(x, w, r, 1e-5, 32, step.rms_norm_quantized(x, w, residual=r, group=32))
    _check_backward(dy, got[1], w, got[2], r, step.rms_norm_backward(dy, got[1], w, got[2], dsummed=r))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("d", [40, 64, 81])
def test_strides(dtype, d):
    """Heads as views of a projection, a broadcast residual, transposed outer sizes, rows off every boundary, and more outer sizes than three."""
    w = _w(d, dtype)
    every = _x((3, 17, 5, 3, d), dtype, 11)
    q, k = every[:, :, :, 0], every[:, :, :, 1]

    def same(x, r):
        """Which terms of a row are added up first goes by where rows begin: within the bounds of any order, not bit for bit."""
        got = step.rms_norm_forward(x, w, residual=r)
        _check_forward(x, w, r, 1e-5, got)
        _check_quantized(x, w, r, 1e-5, 32, step.rms_norm_quantized(x, w, residual=r, group=32))
        for s in (got[1], x):
            _check_backward(x, s, w, got[2], r, step.rms_norm_backward(x, s, w, got[2], dsummed=r))

    same(q, k)
    same(q, k.contiguous())
    same(q.permute(0, 2, 1, 3).contiguous().permute(0, 2, 1, 3), k)
    same(q.permute(2, 1, 0, 3).contiguous().permute(2, 1, 0, 3), k.permute(1, 0, 2, 3).contiguous().permute(1, 0, 2, 3))
    same(q.permute(0, 1, 3, 2).contiguous().permute(0, 1, 3, 2), k)           # a row's elements apart
    off = torch.empty(q.numel() + 1, dtype=dtype, device="cuda")[1:].view(q.shape)
    off.copy_(q)
    same(off, k)
    shared = k[:, :, :1].expand(-1, -1, 5, -1)
    same(q, shared)
    six = every.view(3, 17, 5, 1, 3, d)
    flat = step.rms_norm_forward(every.reshape(-1, d), w)
    got = step.rms_norm_forward(six, w)
    assert got[0].shape == six.shape and torch.equal(got[0].reshape(-1, d), flat[0]) and torch.equal(got[2].reshape(-1), flat[2])
    one = step.rms_norm_forward(q[0, 0, 0], w)
    assert one[2].shape == ()
    o = mo.rms_norm(q[0, 0, 0], w, None, 1e-5)
    mo.close(one[0], o["y"], mo.rounded(o["y"], o["y_off"], dtype))


@pytest.mark.parametrize("d", [8, 96, 1021, 2048, 9000, 40000])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_rows_of_every_size(dtype, d):
    """Squares that 32 bits do not hold, rows of zeros, and rows so small that eps is all there is, or there is none."""
    sizes = [1e37, 1e30, 1e20, 1e10, 1.0, 1e-10, 1e-20, 1e-30, 0.0]
    x = torch.stack([_x((d,), F32, i) * s for i, s in enumerate(sizes)]).clamp(-3e38, 3e38).to(dtype)
    w = _w(d, F32)
    for eps in (1e-5, 0.0, 1e-30):
        rows = x if eps else x[:-1]
        got = step.rms_norm_forward(rows, w, eps=eps)
        _check_forward(rows, w, None, eps, got)
        _check_quantized(rows, w, None, eps, 64, step.rms_norm_quantized(rows, w, eps=eps, group=64))
    y, _, rstd = step.rms_norm_forward(torch.zeros((2, d), dtype=dtype, device="cuda"), w, eps=0.0)
    assert bool(y.isnan().all()) and bool(rstd.isinf().all())
    q, scales, _, _ = step.rms_norm_quantized(torch.zeros((2, d), dtype=dtype, device="cuda"), w)
    assert not bool(q.float().any()) and bool((scales == 2.0 ** -126).all())


@pytest.mark.parametrize("d", [40, 130, 1021, 2048, 40000])
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
def test_infinities_and_nan_stay_in_their_rows(dtype, d):
    x, w = _x((6, d), dtype, 12), _w(d, F32)
    x[1, d // 2], x[3, 0], x[4, d - 1] = float("nan"), float("inf"), float("-inf")
    clean = x.clone()
    clean[[1, 3, 4]] = 0
    y, _, rstd = step.rms_norm_forward(x, w)
    want, _, want_rstd = step.rms_norm_forward(clean, w)
    assert torch.equal(y[[0, 2, 5]], want[[0, 2, 5]]) and torch.equal(rstd[[0, 2, 5]], want_rstd[[0, 2, 5]])
    assert bool(y[1].isnan().all()) and bool(rstd[1].isnan())
    for row, at in ((3, 0), (4, d - 1)):
        assert float(rstd[row]) == 0 and bool(y[row, at].isnan()) and int(y[row].isnan().sum()) == 1 and not bool(y[row].nan_to_num(0.0).any())
    q, scales, _, _ = step.rms_norm_quantized(x, w, group=32)
    assert bool(q[1].float().isnan().all()) and bool(scales[1].isnan().all()) and bool(q[3, 0].float().isnan()) and not bool(scales[3, 1:].isnan().any())
    assert torch.equal(q[[0, 2, 5]].view(torch.uint8), step.rms_norm_quantized(clean, w, group=32)[0][[0, 2, 5]].view(torch.uint8))
    dx, dw = step.rms_norm_backward(x, clean, w, want_rstd)
    fine, _ = step.rms_norm_backward(clean, clean, w, want_rstd)
    assert torch.equal(dx[[0, 2, 5]], fine[[0, 2, 5]])
    # a row of zeros has a normalised part of zero: what dy holds there reaches the row itself and the weight's column alone
    assert bool(dw[d // 2].isnan()) and int((~dw.isfinite()).sum()) == 3


def test_nothing_to_do():
    w = _w(16, BF16)
    x = torch.empty((3, 0, 16), dtype=BF16, device="cuda")
    y, s, rstd = step.rms_norm_forward(x, w, residual=x)
    assert y.shape == s.shape == x.shape and rstd.shape == (3, 0)
    q, scales, _, _ = step.rms_norm_quantized(x, w, group=32)
    assert q.shape == x.shape and scales.shape == (3, 0, 1)
    dx, dw = step.rms_norm_backward(x, x, w, rstd)
    assert dx.shape == x.shape and not bool(dw.any())


def test_offsets_beyond_32_bits():
    d, rows = 8192, 300_000
    x = torch.ones((rows, d), dtype=BF16, device="cuda")
    x[-1] = 2.0
    y, _, rstd = step.rms_norm_forward(x, torch.ones(d, dtype=BF16, device="cuda"), eps=0.0)
    assert float(rstd[-1]) == 0.5 and bool((y[-1] == 1).all()) and bool((y[rows // 2] == 1).all())
    dx, dw = step.rms_norm_backward(y, x, torch.ones(d, dtype=BF16, device="cuda"), rstd)
    assert not bool(dx[-1].any()) and bool((dw.float() == torch.tensor(float(rows), device="cuda").bfloat16().float()).all())


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_gradients(dtype):
    """Through autograd against the formula's in 64 bits, and the formula's against differences."""
    shape, d = (4, 9, 48), 48
    x, r, w = (t.requires_grad_() for t in (_x(shape, dtype, 13), _x(shape, dtype, 14), _w(d, F32)))
    cy, cs = _x(shape, dtype, 15), _x(shape, dtype, 16)
    y, s = step.rms_norm(x, w, residual=r)
    torch.autograd.backward((y, s), (cy, cs))
    rstd = step.rms_norm_forward(x.detach(), w.detach(), residual=r.detach())[2]
    o = mo.rms_norm_backward(cy, s.detach(), w.detach(), rstd, cs)
    mo.close(x.grad, o["dx"], o["dx_bound"])
    mo.close(w.grad, o["dw"], o["dw_bound"])
    assert torch.equal(x.grad, r.grad) and w.grad.dtype == F32
    loss = lambda s, w: ((s * (s.square().mean(-1, keepdim=True) + 1e-5).rsqrt() * w) * cy.double()).sum() + (s * cs.double()).sum()  # noqa: E731
    s64, w64, h = s.detach().double(), w.detach().double(), 1e-5
    way, along = _x(shape, F32, 17).double(), _x((d,), F32, 18).double()
    exact = mo.rms_norm_backward(cy, s64, w64, (s64.square().mean(-1) + 1e-5).rsqrt(), cs)
    slope = (loss(s64 + h * way, w64) - loss(s64 - h * way, w64)) / (2 * h)
    assert math.isclose(float((exact["dx"] * way).sum()), float(slope), rel_tol=1e-6, abs_tol=1e-6)
    slope = (loss(s64, w64 + h * along) - loss(s64, w64 - h * along)) / (2 * h)
    assert math.isclose(float((exact["dw"] * along).sum()), float(slope), rel_tol=1e-6, abs_tol=1e-6)


def test_gradients_where_one_result_is_used():
    x, r, w = (_x((5, 32), F32, 19).requires_grad_(), _x((5, 32), F32, 20).requires_grad_(), _w(32, F32).requires_grad_())
    y, s = step.rms_norm(x, w, residual=r)
    s.sum().backward()
    assert bool((x.grad == 1).all()) and bool((r.grad == 1).all()) and w.grad is None
    x.grad = r.grad = None
    y, s = step.rms_norm(x, w, residual=r)
    y.sum().backward()
    want = step.rms_norm_backward(torch.ones_like(y), s.detach(), w.detach(), step.rms_norm_forward(x.detach(), w.detach(), residual=r.detach())[2])
    assert torch.equal(x.grad, want[0]) and torch.equal(w.grad, want[1])
    z = step.rms_norm(x.detach(), w)
    z.sum().backward(inputs=[w])
    # gradients that arrive broadcast or transposed
    for dy in (y.new_ones(()).expand_as(y), _x((32, 5), F32, 21).t()):
        a, b = (x.detach().clone().requires_grad_() for _ in range(2))
        step.rms_norm(a, w.detach()).backward(dy)
        step.rms_norm(b, w.detach()).backward(dy.contiguous())
        assert torch.equal(a.grad, b.grad)


def test_another_stream():
    x, w = _x((3000, 512), BF16, 22), _w(512, F32)
    y, _, rstd = step.rms_norm_forward(x, w)
    want = step.rms_norm_backward(y, x, w, rstd)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        y2, _, rstd2 = step.rms_norm_forward(x, w)
        got = step.rms_norm_backward(y2, x, w, rstd2)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("what", ["cpu", "dtype", "weight", "weight type", "weight strided", "residual", "residual type", "eps", "nan eps", "group", "no columns", "scalar"])
def test_refusals_forward(what):
    x, w, kw, bad = _x((4, 64), F32, 23), _w(64, F32), {}, hb.ERR_INVALID_ARG
    if what == "cpu":
        x = x.cpu()
    elif what == "dtype":
        x = x.double()
    elif what == "weight":
        w = w[:63]
    elif what == "weight type":
        w = w.double()
    elif what == "weight strided":
        w = _w(128, F32)[::2]
    elif what == "residual":
        kw = dict(residual=x[:3])
    elif what == "residual type":
        kw = dict(residual=x.bfloat16())
    elif what == "eps":
        kw = dict(eps=-1e-5)
    elif what == "nan eps":
        kw = dict(eps=float("nan"))
    elif what == "group":
        kw, bad = dict(group=48), hb.ERR_UNSUPPORTED
    elif what == "no columns":
        x, w = x[:, :0], w[:0]
    elif what == "scalar":
        x = x[0, 0]
    with pytest.raises(hb.HalosError) as e:
        (step.rms_norm_quantized if what == "group" else step.rms_norm_forward)(x, w, **kw)
    assert e.value.status == bad


@pytest.mark.parametrize("what", ["cpu", "summed", "summed type", "rstd", "rstd type", "dsummed", "weight"])
def test_refusals_backward(what):
    dy, s, w, rstd, ds = _x((4, 64), F32, 24), _x((4, 64), F32, 25), _w(64, F32), torch.ones(4, device="cuda"), None
    if what == "cpu":
        dy = dy.cpu()
    elif what == "summed":
        s = s[:3]
    elif what == "summed type":
        s = s.half()
    elif what == "rstd":
        rstd = rstd[:3]
    elif what == "rstd type":
        rstd = rstd.double()
    elif what == "dsummed":
        ds = s[:, :63]
    elif what == "weight":
        w = w.cpu()
    with pytest.raises(hb.HalosError) as e:
        step.rms_norm_backward(dy, s, w, rstd, dsummed=ds)
    assert e.value.status == hb.ERR_INVALID_ARG
