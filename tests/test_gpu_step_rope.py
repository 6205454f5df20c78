"""Rotary positions against the 64-bit form: layouts, partly rotated heads, odd widths, strides, positions far out."""
from __future__ import annotations

import math
from fractions import Fraction

import pytest
import torch

import step_oracle as so
from paper_2506_04531_b200 import binding as hb, step

pytestmark = pytest.mark.gpu


def _x(shape, dtype, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(shape, generator=g, device="cuda").to(dtype)


def _close(got, want, bound, dtype):
    off = (got.double() - want).abs()
    allowed = bound + (so.U[dtype] * want.abs() + so.TINY[dtype] if dtype != torch.float32 else 0)
    assert bool((off <= allowed).all()), float((off - allowed).max())


@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("b,s,hq,hk,d,rot", [(1, 1, 1, 1, 2, 2), (2, 7, 3, 1, 64, 16), (3, 33, 12, 12, 64, 64), (1, 130, 5, 5, 80, 20), (2, 9, 4, 2, 128, 96), (1, 5, 2, 2, 256, 256),
                                              (2, 3, 3, 1, 7, 6), (1, 4, 2, 1, 17, 10), (1, 2, 33, 33, 40, 24)])
def test_against_64_bits(b, s, hq, hk, d, rot, dtype, layout):
    q, k = _x((b, s, hq, d), dtype, 1), _x((b, s, hk, d), dtype, 2)
    freqs, mag = step.rotary_frequencies(rot, scaling="ramp", factor=4.0)
    pos = torch.randint(0, 5000, (b, s), device="cuda", generator=torch.Generator(device="cuda").manual_seed(3), dtype=torch.int32)
    for inverse in (False, True):
        q2, k2 = step.rope(q, k, freqs, positions=pos, layout=layout, magnitude=mag, inverse=inverse)
        for x, y in ((q, q2), (k, k2)):
            want, bound = so.rope(x, freqs, pos, layout, mag, inverse)
            _close(y, want, bound, dtype)
            assert torch.equal(y[..., rot:], x[..., rot:])


@pytest.mark.parametrize("base", [0, 2047, 2 ** 24 + 1, 10 ** 9 + 7, 2 ** 31 + 5, -12345])
def test_far_positions_are_as_exact_as_near_ones(base):
    q = _x((2, 5, 2, 64), torch.float32, 4)
    freqs, _ = step.rotary_frequencies(64)
    pos = torch.arange(5, device="cuda")[None].expand(2, -1) + base
    want, bound = so.rope(q, freqs, pos, "half", 1.0, False)
    y, none = step.rope(q, None, freqs, positions=pos)
    assert none is None
    _close(y, want, bound, torch.float32)
    y2, _ = step.rope(q, None, freqs, offset=base)
    assert torch.equal(y, y2)
    if -2 ** 31 <= base < 2 ** 31 - 5:
        assert torch.equal(y, step.rope(q, None, freqs, positions=pos.to(torch.int32))[0])
    assert torch.equal(y, step.rope(q, None, freqs, positions=pos[0])[0])


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_strides_views_and_in_place(dtype):
    freqs, _ = step.rotary_frequencies(16)
    fused = _x((2, 19, 6, 3, 64), dtype, 5)
    q, k = fused[:, :, :, 0], fused[:, :, :, 1]
    want = step.rope(q.contiguous(), k.contiguous(), freqs, offset=3)
    got = step.rope(q, k, freqs, offset=3)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    heads_first = q.permute(0, 2, 1, 3).contiguous().permute(0, 2, 1, 3)
    assert torch.equal(step.rope(heads_first, None, freqs, offset=3)[0], want[0])
    shared = k[:, :, :1].expand(-1, -1, 6, -1)                  # a broadcast head
    assert torch.equal(step.rope(shared, None, freqs, offset=3)[0], step.rope(shared.contiguous(), None, freqs, offset=3)[0])
    off = torch.empty(q.numel() + 1, dtype=dtype, device="cuda")[1:].view(q.shape)   # off every vector boundary
    off.copy_(q)
    assert torch.equal(step.rope(off, None, freqs, offset=3)[0], want[0])
    with pytest.raises(hb.HalosError):
        step.rope(shared, None, freqs, inplace=True)
    before = fused.clone()
    step.rope(q, k, freqs, offset=3, inplace=True)
    assert torch.equal(q, want[0]) and torch.equal(k, want[1]) and torch.equal(fused[:, :, :, 2], before[:, :, :, 2])


def test_gradient_against_the_form_and_against_differences():
    q, k = _x((2, 11, 4, 32), torch.float32, 6).requires_grad_(), _x((2, 11, 2, 32), torch.float32, 7).requires_grad_()
    freqs, mag = step.rotary_frequencies(24, scaling="ramp", factor=8.0)
    pos = torch.arange(11, device="cuda")[None].expand(2, -1) * 37
    wq, wk = _x(q.shape, torch.float32, 8), _x(k.shape, torch.float32, 9)
    a, b = step.rotary(q, k, freqs, positions=pos, layout="interleaved", magnitude=mag)
    ((a * wq).sum() + (b * wk).sum()).backward()
    loss = lambda x: (so.rope(x, freqs, pos, "interleaved", mag, False)[0] * wq.double()).sum()  # noqa: E731
    want, bound = so.rope(wq, freqs, pos, "interleaved", mag, True)
    _close(q.grad, want, bound, torch.float32)
    way = _x(q.shape, torch.float32, 10).double()
    slope = (loss(q.detach().double() + way) - loss(q.detach().double() - way)) / 2      # linear: any step will do
    assert abs(float((q.grad.double() * way).sum() - slope)) <= float((bound * way.abs()).sum())
    assert torch.equal(k.grad, step.rope(wk, None, freqs, positions=pos, layout="interleaved", magnitude=mag, inverse=True)[0])


def test_empty_and_other_stream():
    freqs, _ = step.rotary_frequencies(8)
    assert step.rope(torch.empty(0, 5, 2, 8, device="cuda"), None, freqs)[0].shape == (0, 5, 2, 8)
    assert step.rope(torch.empty(2, 0, 2, 8, device="cuda"), None, freqs)[0].shape == (2, 0, 2, 8)
    q = _x((4, 300, 8, 8), torch.float32, 11)
    want = step.rope(q, None, freqs)[0]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        got = step.rope(q, None, freqs)[0]
    side.synchronize()
    assert torch.equal(got, want)


def test_frequencies():
    w, one = step.rotary_frequencies(8, device="cpu")
    assert one == 1.0 and torch.allclose(w, torch.tensor([10000.0 ** (-p / 4) for p in range(4)], dtype=torch.float64))
    assert torch.equal(step.rotary_frequencies(8, scaling="linear", factor=4.0, device="cpu")[0] * 4, w)
    v, _ = step.rotary_frequencies(8, scaling="base", factor=4.0, device="cpu")
    assert float(v[0]) == 1.0 and math.isclose(float(v[-1]), float(w[-1]) / 4, rel_tol=1e-12)
    v, mag = step.rotary_frequencies(128, scaling="ramp", factor=4.0, device="cpu")
    w, _ = step.rotary_frequencies(128, device="cpu")
    assert float(v[0]) == float(w[0]) and math.isclose(float(v[-1]), float(w[-1]) / 4, rel_tol=1e-12) and mag > 1
    assert bool((v[1:] < v[:-1]).all())


@pytest.mark.parametrize("what", ["cpu", "dtype", "layout", "odd", "wide", "freqs", "positions", "strided", "shape"])
def test_refusals(what):
    q, freqs, kw = _x((1, 4, 2, 16), torch.float32, 12), step.rotary_frequencies(8)[0], {}
    k = None
    if what == "cpu":
        q = q.cpu()
    elif what == "dtype":
        q = q.double()
    elif what == "layout":
        kw = dict(layout="thirds")
    elif what == "odd":
        freqs = torch.ones(9, dtype=torch.float64, device="cuda")        # 18 of 16 elements
    elif what == "wide":
        q = _x((1, 1, 1, 264), torch.float32, 12)
    elif what == "freqs":
        freqs = freqs.float()
    elif what == "positions":
        kw = dict(positions=torch.zeros(5, dtype=torch.int32, device="cuda"))
    elif what == "strided":
        q = _x((1, 4, 2, 32), torch.float32, 12)[..., ::2]
    elif what == "shape":
        k = _x((1, 5, 2, 16), torch.float32, 12)
    with pytest.raises(hb.HalosError) as e:
        step.rope(q, k, freqs, **kw)
    assert e.value.status in (hb.ERR_INVALID_ARG, hb.ERR_UNSUPPORTED)


def test_gradient_without_keys():
    q = _x((2, 5, 3, 32), torch.float32, 13).requires_grad_()
    freqs, w = step.rotary_frequencies(24)[0], _x(q.shape, torch.float32, 14)
    y, none = step.rotary(q, None, freqs, offset=7)
    assert none is None
    (y * w).sum().backward()
    assert torch.equal(q.grad, step.rope(w, None, freqs, offset=7, inverse=True)[0])


# 2 pi to 60 digits: what a 64-bit float leaves out of it is 10^-4 of a turn at position 2^40
TWO_PI = Fraction(6283185307179586476925286766559005768394338798750211641949889, 10 ** 60)


@pytest.mark.parametrize("base", [0, 10 ** 6 + 3, 2 ** 31 - 40, -2 ** 31, 2 ** 36 + 1, 2 ** 40 + 12345, -2 ** 44])
def test_angles_against_exact_ones(base):
    """Ones and zeros, so that cosine and sine of the angles come back as they are."""
    freqs, seq = step.rotary_frequencies(64, scaling="linear", factor=3.0)[0], 33
    q = torch.zeros((1, seq, 1, 64), device="cuda")
    q[..., :32] = 1.0
    y = step.rope(q, None, freqs, offset=base)[0][0, :, 0].double().cpu()
    turns = [[float(Fraction(w) * (base + s) / TWO_PI % 1) for w in freqs.tolist()] for s in range(seq)]
    angle = torch.tensor(turns, dtype=torch.float64) * (2 * math.pi)
    # the angle: 2^-31 of a turn, 2^-62 more for each position, 2^-25 half turns of rounding; sine and cosine 2 ulp, rounded once more
    bound = (2.0 ** -31 + 2.0 ** -62 * abs(base)) * 2 * math.pi + 2.0 ** -25 * math.pi + 3 * 2.0 ** -24
    assert float((y[:, :32] - angle.cos()).abs().max()) <= bound
    assert float((y[:, 32:] - angle.sin()).abs().max()) <= bound
