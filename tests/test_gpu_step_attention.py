"""Attention, forward and backward, against the 64-bit form: sizes around the tiles' edges, masks that leave rows empty, what lies in masked
places, shared heads, strides, and gradients against differences."""
from __future__ import annotations

import math

import pytest
import torch

import step_oracle as so
from paper_2506_04531_b200 import binding as hb, step

pytestmark = pytest.mark.gpu

BF16, F16 = torch.bfloat16, torch.float16


def _x(shape, dtype, seed, scale=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(shape, generator=g, device="cuda") * scale).to(dtype)


def _within(got, want, bound, what):
    assert bool(torch.isfinite(got).all()), what
    off = (got.double() - want).abs()
    assert bool((off <= bound).all()), (what, float((off - bound).max()))


def _check(q, k, v, dout, scale=None, **mask):
    scale = q.shape[3] ** -0.5 if scale is None else scale
    o, lse = step.attention_forward(q, k, v, scale=scale, **mask)
    grads = step.attention_backward(dout, q, k, v, o, lse, scale=scale, **mask)
    want = so.attention(q, k, v, dout, scale=scale, **{"causal": True, **mask})
    _within(o, want["o"], want["o_bound"], "o")
    none = want["lse"] == -math.inf
    assert torch.equal(lse == -math.inf, none)
    assert bool(((lse.double() - want["lse"])[~none].abs() <= 1e-5 * (1 + want["lse"][~none].abs())).all())
    for name, got in zip(("dq", "dk", "dv"), grads):
        _within(got, want[name], want[name + "_bound"], name)
    assert not step.fault()
    return o, lse, grads


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("d", [8, 64, 72, 128])
@pytest.mark.parametrize("s", [1, 2, 63, 64, 65, 127, 128, 129, 300])
def test_causal_lengths(s, d, dtype):
    q, k, v, do = (_x((2, s, 2, d), dtype, i) for i in range(4))
    _check(q, k, v, do)


@pytest.mark.parametrize("dtype,d", [(BF16, 64), (F16, 128)])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("sq,sk", [(1, 1), (1, 700), (5, 130), (130, 5), (200, 257), (257, 200), (129, 1)])
def test_queries_and_keys_of_different_lengths(sq, sk, causal, dtype, d):
    q, do = _x((1, sq, 4, d), dtype, 1), _x((1, sq, 4, d), dtype, 2)
    k, v = _x((1, sk, 2, d), dtype, 3), _x((1, sk, 2, d), dtype, 4)
    _check(q, k, v, do, causal=causal)      # causal with sq > sk: the first rows see nothing


@pytest.mark.parametrize("dtype,d", [(BF16, 64), (F16, 64), (BF16, 128)])
@pytest.mark.parametrize("heads,kv", [(1, 1), (6, 2), (8, 1), (5, 5)])
def test_shared_heads(heads, kv, dtype, d):
    q, do = _x((2, 150, heads, d), dtype, 1), _x((2, 150, heads, d), dtype, 2)
    k, v = _x((2, 150, kv, d), dtype, 3), _x((2, 150, kv, d), dtype, 4)
    _check(q, k, v, do)
    _check(q, k, v, do, causal=False, scale=0.3)


@pytest.mark.parametrize("garbage", [float("nan"), float("inf"), -3e38])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("d", [64, 96])
def test_lengths_with_anything_past_the_end(d, causal, garbage):
    s, lens = 270, [270, 0, 1, 64, 65, 128, 200, 5]
    q, k, v, do = (_x((len(lens), s, 3, d), BF16, i) for i in range(4))
    for b, n in enumerate(lens):
        for x in (q, k, v, do):
            x[b, n:] = garbage
    _check(q, k, v, do, causal=causal, lens=torch.tensor(lens, dtype=torch.int32, device="cuda"))


@pytest.mark.parametrize("dtype,d", [(BF16, 64), (F16, 128)])
def test_documents(dtype, d):
    s = 333
    starts = torch.zeros((2, s), dtype=torch.int32, device="cuda")
    for b, cuts in enumerate(([0, 1, 2, 3, 64, 129, 130, 300], [0, 127, 128, 256])):
        for c in cuts:
            starts[b, c:] = c
    q, do = _x((2, s, 4, d), dtype, 1), _x((2, s, 4, d), dtype, 2)
    k, v = _x((2, s, 2, d), dtype, 3), _x((2, s, 2, d), dtype, 4)
    _check(q, k, v, do, doc_start=starts)
    _check(q, k, v, do, doc_start=starts, lens=torch.tensor([s, 140], dtype=torch.int32, device="cuda"))
    _check(q, k, v, do, doc_start=starts, causal=False)


def test_rows_that_see_nothing_may_hold_anything():
    """Left padding: the first rows of a sequence see nothing, and nobody sees them."""
    s, pad = 200, 70
    q, k, v, do = (_x((1, s, 2, 64), BF16, i) for i in range(4))
    for x in (q, k, v, do):
        x[:, :pad] = float("nan")
    starts = torch.full((1, s), pad, dtype=torch.int32, device="cuda")
    o, lse, (dq, dk, dv) = _check(q, k, v, do, doc_start=starts)
    assert float(o[:, :pad].abs().sum()) == 0 and bool((lse[..., :pad] == -math.inf).all())
    assert all(float(x[:, :pad].abs().sum()) == 0 for x in (dq, dk, dv))


def test_one_visible_key_gives_no_gradient_to_queries_and_keys():
    q, k, v, do = (_x((3, 1, 4, 64), BF16, i) for i in range(4))
    o, lse, (dq, dk, dv) = _check(q, k, v, do)
    assert torch.equal(o, v) and float(dq.abs().sum()) == float(dk.abs().sum()) == 0 and torch.equal(dv, do)


@pytest.mark.parametrize("spread", [12.0, 40.0])
def test_large_scores(spread):
    """Sharp rows: the running maximum moves late and far."""
    q, k = _x((1, 600, 2, 64), BF16, 1, spread), _x((1, 600, 2, 64), BF16, 2)
    k[:, 500:] *= 4
    v, do = _x((1, 600, 2, 64), BF16, 3), _x((1, 600, 2, 64), BF16, 4)
    want = so.attention(q, k, v, None, scale=0.125, causal=False)
    o, lse = step.attention_forward(q, k, v, causal=False)
    # scores of size s are formed in 32 bits: off by 2^-23 s in the exponent
    more = float((q.double().abs().amax() * k.double().abs().amax() * 64 * 0.125)) * 2.0 ** -22
    assert bool(((o.double() - want["o"]).abs() <= want["o_bound"] + more * v.double().abs().max()).all())
    assert bool(((lse.double() - want["lse"]).abs() <= 1e-5 + 2.0 ** -22 * want["lse"].abs()).all())


def test_strides_orders_and_broadcast_heads():
    fused = _x((2, 140, 4, 3, 64), BF16, 1)
    q, k, v = (fused[:, :, :, i] for i in range(3))
    do = _x((2, 140, 4, 64), BF16, 2)
    plain = [x.contiguous() for x in (q, k, v)]
    o, lse, grads = _check(*plain, do)
    same = lambda a: torch.equal(a[0], o) and torch.equal(a[1], lse) and all(torch.equal(x, y) for x, y in zip(a[2], grads))  # noqa: E731
    assert same(_check(q, k, v, do))
    heads_first = [x.permute(0, 2, 1, 3).contiguous().permute(0, 2, 1, 3) for x in (*plain, do)]
    assert same(_check(*heads_first))
    off = []
    for x in (*plain, do):                                        # off every 16-byte boundary
        y = torch.empty(x.numel() + 1, dtype=x.dtype, device="cuda")[1:].view(x.shape)
        off.append(y.copy_(x))
    assert same(_check(*off))
    one = plain[1][:, :, :1].expand(-1, -1, 4, -1)
    a, b = _check(plain[0], one, one, do), _check(plain[0], one.contiguous(), one.contiguous(), do)
    assert torch.equal(a[0], b[0]) and all(torch.equal(x, y) for x, y in zip(a[2], b[2]))
    # a broadcast input through autograd: its gradient is the sum over the heads that read it
    leaf = plain[1][:, :, :1].clone().requires_grad_()
    step.attention(plain[0], leaf.expand(-1, -1, 4, -1), plain[2], causal=True).backward(do)
    want = so.attention(plain[0], leaf.detach(), plain[2][:, :, :1].expand(-1, -1, 1, -1), None, scale=0.125, causal=True)
    full = so.attention(plain[0], one, plain[2], do, scale=0.125, causal=True)
    assert want["o"].shape == full["o"].shape
    summed, bound = full["dk"].sum(2, keepdim=True), full["dk_bound"].sum(2, keepdim=True)
    assert bool(((leaf.grad.double() - summed).abs() <= bound + 4 * so.U[BF16] * full["dk"].abs().sum(2, keepdim=True)).all())


def test_same_bits_every_time_and_on_another_stream():
    q, k, v, do = (_x((3, 500, 4, 64), BF16, i) for i in range(4))
    run = lambda: (lambda o, l: (o, l, *step.attention_backward(do, q, k, v, o, l)))(*step.attention_forward(q, k, v))  # noqa: E731
    first = run()
    for _ in range(5):
        assert all(torch.equal(a, b) for a, b in zip(first, run()))
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        other = run()
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(first, other))


@pytest.mark.parametrize("b,s,h,kv,d,dtype", [(2, 2048, 12, 12, 64, BF16), (1, 3000, 8, 2, 64, F16), (2, 2048, 8, 8, 128, BF16), (1, 3000, 8, 4, 128, F16)])
def test_same_bits_where_many_tiles_are_under_way(b, s, h, kv, d, dtype):
    """A warp that is ahead of the others must not be counted for one that is behind: this shows in some of many runs of many tiles."""
    q, do = _x((b, s, h, d), dtype, 1), _x((b, s, h, d), dtype, 2)
    k, v = _x((b, s, kv, d), dtype, 3), _x((b, s, kv, d), dtype, 4)
    for causal in (True, False):
        o, lse = step.attention_forward(q, k, v, causal=causal)
        grads = step.attention_backward(do, q, k, v, o, lse, causal=causal)
        assert all(bool(torch.isfinite(x).all()) for x in (o, lse, *grads))
        for _ in range(20):
            assert torch.equal(o, step.attention_forward(q, k, v, causal=causal)[0])
            assert all(torch.equal(x, y) for x, y in zip(grads, step.attention_backward(do, q, k, v, o, lse, causal=causal)))


@pytest.mark.parametrize("dtype,d", [(BF16, 64), (F16, 80), (BF16, 128)])
def test_gradients_against_differences(dtype, d):
    """The slope of sum(o * w) along a random direction, from the 64-bit forward alone, against the kernels' gradients."""
    s = 37
    q, k, v, w = (_x((1, s, 2, d), dtype, i) for i in range(4))
    leaves = [x.clone().requires_grad_() for x in (q, k, v)]
    step.attention(*leaves).backward(w)
    full = so.attention(q, k, v, w, scale=d ** -0.5, causal=True)
    loss = lambda *x: (so_forward(*x, d) * w.double()).sum()  # noqa: E731
    for i, name in enumerate(("dq", "dk", "dv")):
        way, h = _x(q.shape, torch.float32, 20 + i).double(), 1e-4
        at = [x.double() for x in (q, k, v)]
        up, down = list(at), list(at)
        up[i], down[i] = at[i] + h * way, at[i] - h * way
        slope = float((loss(*up) - loss(*down)) / (2 * h))
        allowed = float((full[name + "_bound"] * way.abs()).sum()) + 1e-5 * abs(slope)
        assert abs(float((leaves[i].grad.double() * way).sum()) - slope) <= allowed, name


def so_forward(q, k, v, d):
    """o [1, s, h, d] in 64 bits, causal."""
    s = torch.einsum("bihd,bjhd->bhij", q, k) * d ** -0.5
    n = s.shape[-1]
    s = s.masked_fill(torch.ones(n, n, device=s.device).triu(1).bool(), -math.inf)
    return torch.einsum("bhij,bjhd->bihd", torch.softmax(s, -1), v)


def test_empty_sizes():
    z = lambda *s: torch.zeros(s, dtype=BF16, device="cuda")  # noqa: E731
    o, lse = step.attention_forward(z(0, 5, 2, 64), z(0, 5, 2, 64), z(0, 5, 2, 64))
    assert o.shape == (0, 5, 2, 64) and lse.shape == (0, 2, 5)
    o, lse = step.attention_forward(z(1, 0, 2, 64), z(1, 5, 2, 64), z(1, 5, 2, 64))
    assert o.shape == (1, 0, 2, 64)
    k = _x((1, 5, 2, 64), BF16, 1)
    _, dk, dv = step.attention_backward(z(1, 0, 2, 64), z(1, 0, 2, 64), k, k, o, lse)
    assert float(dk.abs().sum()) == float(dv.abs().sum()) == 0
    q = _x((1, 3, 2, 64), BF16, 2)
    o, lse = step.attention_forward(q, z(1, 0, 2, 64), z(1, 0, 2, 64))      # no keys at all
    assert float(o.abs().sum()) == 0 and bool((lse == -math.inf).all())
    dq, dk, _ = step.attention_backward(q, q, z(1, 0, 2, 64), z(1, 0, 2, 64), o, lse)
    assert float(dq.abs().sum()) == 0 and dk.shape == (1, 0, 2, 64)


@pytest.mark.parametrize("what,status", [("f32", hb.ERR_UNSUPPORTED), ("d", hb.ERR_UNSUPPORTED), ("wide", hb.ERR_UNSUPPORTED), ("heads", hb.ERR_INVALID_ARG), ("scale", hb.ERR_INVALID_ARG),
                                         ("mixed", hb.ERR_INVALID_ARG), ("shape", hb.ERR_INVALID_ARG), ("cpu", hb.ERR_INVALID_ARG), ("lens", hb.ERR_INVALID_ARG), ("starts", hb.ERR_INVALID_ARG)])
def test_refusals(what, status):
    d = {"d": 60, "wide": 136}.get(what, 64)
    dtype = torch.float32 if what == "f32" else BF16
    q, k, v = (_x((1, 8, 3 if i == 0 else 2 if what == "heads" else 3, d), dtype, i) for i in range(3))
    kw = {}
    if what == "scale":
        kw = dict(scale=-1.0)
    elif what == "mixed":
        k = k.half()
    elif what == "shape":
        v = v[:, :5]
    elif what == "cpu":
        k = k.cpu()
    elif what == "lens":
        kw = dict(lens=torch.zeros(1, dtype=torch.int64, device="cuda"))
    elif what == "starts":
        kw = dict(doc_start=torch.zeros(8, dtype=torch.int32, device="cuda"))
    with pytest.raises(hb.HalosError) as e:
        step.attention_forward(q, k, v, **kw)
    assert e.value.status == status
