"""Attention where scores or gradients are far from 1: the kernels end, and what can be right in 32 bits is."""
from __future__ import annotations


import pytest
import torch

import step_oracle as so
from paper_2506_04531_b200 import binding as hb, step

pytestmark = pytest.mark.gpu

BF16, F16 = torch.bfloat16, torch.float16


def _x(shape, dtype, seed, scale=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(shape, generator=g, device="cuda") * scale).to(dtype)


def _check_forward(q, k, v, scale, causal):
    """Equal keys have equal scores whatever those are, and so probabilities of the bounds' accuracy."""
    o, lse = step.attention_forward(q, k, v, scale=scale, causal=causal)
    want = so.attention(q, k, v, None, scale=scale, causal=causal)
    assert bool(((o.double() - want["o"]).abs() <= want["o_bound"]).all())
    # a score is a sum in 32 bits, off by 2^-20 of its terms' sizes at worst, and lse three roundings of it
    terms = torch.einsum("bihd,bjhd->bhij", q.double().abs(), k.double().abs()).amax(-1) * scale
    assert bool(((lse.double() - want["lse"]).abs() <= 2.0 ** -20 * terms + 2.0 ** -22 * want["lse"].abs() + 1e-5).all())
    assert not step.fault()


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("power", [10, 20, 24, 27, 28, 29, 30])
def test_equal_keys_with_large_scores(power, causal, d, dtype):
    """Scores of some 2^power of either sign: a token that is repeated, in a run that has diverged."""
    if dtype == F16 and power == 30:
        pytest.skip("float16 does not hold these inputs")
    q = _x((1, 300, 2, d), dtype, power, 2.0 ** (power / 2 - 1))
    k = _x((1, 1, 2, d), dtype, power + 1, 2.0 ** (power / 2 - 1)).expand(-1, 300, -1, -1)
    _check_forward(q, k, _x((1, 300, 2, d), dtype, 3), d ** -0.5, causal)


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("late", [0, 63, 64, 200, 299])
@pytest.mark.parametrize("power", [16, 24, 28, 30])
def test_one_key_far_above_the_others(power, late, dtype):
    """Rows whose maximum goes from small to large at a late key, or is large from the first key on."""
    q = _x((1, 300, 2, 64), dtype, 1).abs() + 0.5
    k = _x((1, 300, 2, 64), dtype, 2)
    k[:, late] = 2.0 ** (power / 2)
    _check_forward(q * 2.0 ** (power / 2 - 6), k * 2.0 ** -6, _x((1, 300, 2, 64), dtype, 3), 2.0 ** 6, False)


@pytest.mark.parametrize("scale", [2.0 ** 24, 2.0 ** 30, 2.0 ** 60, 2.0 ** 100])
@pytest.mark.parametrize("sign", [1.0, -1.0])
def test_large_scale(sign, scale):
    """Equal keys again, so that a row is the mean of the values so far; 64 bits would not hold log sum exp of the larger ones."""
    q, k, v = _x((1, 200, 2, 64), BF16, 1) * sign, _x((1, 1, 2, 64), BF16, 2).expand(-1, 200, -1, -1), _x((1, 200, 2, 64), BF16, 3)
    o, lse = step.attention_forward(q, k, v, scale=scale)
    seen = torch.arange(1, 201, dtype=torch.float64, device="cuda")[None, :, None, None]
    want, spread = v.double().cumsum(1) / seen, v.double().abs().cumsum(1) / seen
    assert bool(((o.double() - want).abs() <= (so.U[BF16] + 4e-6) * spread + so.U[BF16] * want.abs()).all())
    score = scale * torch.einsum("bihd,bjhd->bhij", q.double(), k[:, :1].double())[..., 0]
    terms = scale * torch.einsum("bihd,bjhd->bhij", q.double().abs(), k[:, :1].double().abs())[..., 0]
    assert bool(((lse.double() - score - seen[0, :, 0, 0].log()).abs() <= 2.0 ** -20 * terms + 2.0 ** -22 * score.abs() + 1e-5).all())


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("power", [20, 27, 28, 29, 30])
def test_large_scores_of_any_kind_end_in_means_of_the_values(power, dtype):
    """With different keys 32 bits do not say which of two close scores is the larger, but a mean of values lies between them; rows of
    ordinary scores, in the same warps as the others, keep their accuracy."""
    q, k, v = _x((2, 400, 2, 64), dtype, 1), _x((2, 400, 2, 64), dtype, 2), _x((2, 400, 2, 64), dtype, 3)
    q[:, ::2] = (q[:, ::2].float() * 2.0 ** (power - 14)).to(dtype) if dtype == BF16 else q[:, ::2] * 2.0 ** 13
    scale = 0.125 if dtype == BF16 else 0.125 * 2.0 ** (power - 27)
    q[:, 1::2] *= 0.125 / scale
    o, lse = step.attention_forward(q, k, v, scale=scale, causal=False)
    assert bool(torch.isfinite(o).all()) and bool(torch.isfinite(lse).all()) and not step.fault()
    # p and o are rounded once each, and the sum of p is not
    low, high, off = v.amin(1, keepdim=True).double(), v.amax(1, keepdim=True).double(), (1 + so.U[dtype]) ** 2 * (1 + 4e-6) - 1
    assert bool((o.double() >= low - off * low.abs()).all()) and bool((o.double() <= high + off * high.abs()).all())
    want = so.attention(q[:, 1::2], k, v, None, scale=scale, causal=False)
    assert bool(((o[:, 1::2].double() - want["o"]).abs() <= want["o_bound"]).all())


def test_a_scale_that_overflows_is_refused():
    q = _x((1, 8, 1, 64), BF16, 1)
    with pytest.raises(hb.HalosError) as e:
        step.attention_forward(q, q, q, scale=3e38)
    assert e.value.status == hb.ERR_INVALID_ARG


def _gradients(q, k, v, dout, **mask):
    o, lse = step.attention_forward(q, k, v, **mask)
    return step.attention_backward(dout, q, k, v, o, lse, **mask)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("s,causal", [(2048, False), (300, True), (40, True)])
@pytest.mark.parametrize("power", [-16, -14, -10, -6, 6, 10, 12])
def test_gradients_follow_the_size_of_dout_in_float16(power, s, causal, d):
    """dout 2^power times gives gradients 2^power times, but for their own rounding: nothing on the way is too small or too large for the type."""
    q, k, v = (_x((1, s, 2, d), F16, i, 0.5 if i < 2 else 1.0) for i in range(3))
    dout = (_x((1, s, 2, d), torch.float32, 3).clamp(-4, 4) * 16).round().div(16).to(F16)   # multiples of 2^-4: exact at every power here
    one = _gradients(q, k, v, dout, causal=causal)
    other = _gradients(q, k, v, dout * 2.0 ** power, causal=causal)
    for a, b in zip(one, other):
        want = a.double() * 2.0 ** power
        off = 2 * so.U[F16] * want.abs() + 2.0 ** -25 * (1 + 2.0 ** power)
        fits = want.abs() < 65000
        assert bool(((b.double() - want).abs() <= off)[fits].all())


@pytest.mark.parametrize("size", [2.0 ** -10, 30.0, 2000.0])
def test_gradients_follow_the_size_of_the_values_in_float16(size):
    q, k, v, dout = (_x((1, 260, 4, 64), F16, i) for i in range(4))
    dout, v = dout * 2.0 ** -4, v[:, :, :2] * size
    want = so.attention(q, k[:, :, :2], v, dout, scale=0.125, causal=True)
    for name, got in zip(("dq", "dk", "dv"), _gradients(q, k[:, :, :2], v, dout)):
        assert bool(((got.double() - want[name]).abs() <= want[name + "_bound"]).all()), name


@pytest.mark.parametrize("garbage", [float("nan"), float("inf"), -60000.0])
def test_what_nobody_sees_does_not_weigh_on_the_gradients_in_float16(garbage):
    """Past the ends of sequences and before the first document: the same bits as with zeros there."""
    s, lens = 270, torch.tensor([270, 0, 65, 130], dtype=torch.int32, device="cuda")
    starts = torch.zeros((4, s), dtype=torch.int32, device="cuda")
    starts[3] = 70
    q, k, v, dout = (_x((4, s, 4, 64), F16, i) for i in range(4))
    k, v = k[:, :, :2].contiguous(), v[:, :, :2].contiguous()
    place = torch.arange(s, device="cuda")[None]
    unseen = (place >= lens[:, None]) | (place < starts[:, :1])
    fill = lambda x: [t.masked_fill(unseen[:, :, None, None], x) for t in (q, k, v, dout)]  # noqa: E731
    clean, dirty = (_gradients(*fill(x), doc_start=starts, lens=lens) for x in (0.0, garbage))
    assert all(torch.equal(a, b) and bool(torch.isfinite(b).all()) for a, b in zip(clean, dirty))


def test_no_gradient_at_all_in_float16():
    q, k, v = (_x((1, 100, 2, 64), F16, i) for i in range(3))
    for dout, values in ((torch.zeros_like(q), v), (q, torch.zeros_like(v))):
        dq, dk, dv = _gradients(q, k, values, dout)
        assert float(dq.abs().sum()) == float(dk.abs().sum()) == 0
        assert bool(torch.isfinite(dv).all()) and (float(dv.abs().sum()) > 0) == bool(dout.any())
