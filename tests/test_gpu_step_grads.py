"""The norm of many gradients, clipping and the step against 64 bits: types side by side, sizes, strides, and values that 32 bits do not hold squared."""
from __future__ import annotations

import math

import pytest
import torch

import step_more_oracle as mo
from paper_2506_04531_b200 import binding as hb, step

pytestmark = pytest.mark.gpu
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
TYPES = (F32, BF16, F16)


def _x(shape, dtype, seed, scale=1.0):
    return (torch.randn(shape, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda") * scale).to(dtype)


def _check_norm(got, grads):
    want = mo.norm(grads)
    assert got.dtype == F32 and got.shape == () and abs(float(got) - want) <= mo.NORM_OFF * want, (float(got), want)
    return want


def _check_clipped(out, grads, factor):
    for o, g in zip(out, grads):
        want = g.double() * factor
        mo.close(o, want, mo.rounded(want, 8 * mo.E * want.abs(), o.dtype))


SETS = [[(1,)], [(5, 7)], [(0,), (3,), (0, 4)], [(8192,), (8193,), (16384,), (16391,), (1,), (255,)], [(100, 1000), (1000,), (17, 3, 5), (), (300_001,)]]


@pytest.mark.parametrize("shapes", SETS)
@pytest.mark.parametrize("first", range(3))
def test_against_64_bits(shapes, first):
    """Every pair of types comes up."""
    grads = [_x(s, TYPES[(first + i) % 3], i, 0.1) for i, s in enumerate(shapes)]
    norm = _check_norm(step.grad_norm(grads), grads)
    for limit in (norm / 3, norm * 2, 0.0):
        factor = min(1.0, limit / norm)
        for turn in range(3):
            out = [torch.full(g.shape, 7.0, dtype=TYPES[(first + i * 2 + turn) % 3], device="cuda") for i, g in enumerate(grads)]
            _check_norm(step.clip_grads(grads, limit, out=out), grads)
            _check_clipped(out, grads, factor)
            params = [_x(g.shape, o.dtype, 50 + i) for i, (g, o) in enumerate(zip(grads, out))]
            before = [p.clone() for p in params]
            _check_norm(step.sgd_step(params, grads, 0.25, max_norm=limit), grads)
            for p, b, g in zip(params, before, grads):
                moved = 0.25 * factor * g.double()
                want = b.double() - moved
                mo.close(p, want, mo.rounded(want, 9 * mo.E * moved.abs() + mo.E * want.abs(), p.dtype))
        mine = [g.clone() for g in grads]
        _check_norm(step.clip_grads(mine, limit), grads)
        _check_clipped(mine, grads, factor)
        if factor == 1:
            assert all(torch.equal(a, b) for a, b in zip(mine, grads))


def test_a_step_without_a_norm():
    p, g = _x((1000, 33), F32, 1), _x((1000, 33), BF16, 2)
    want = p.double() - 0.5 * g.double()
    assert step.sgd_step([p], [g], 0.5) is None
    mo.close(p, want, mo.rounded(want, mo.E * want.abs() + 2 * mo.E * g.double().abs(), F32))


@pytest.mark.parametrize("count", [31, 33, 320, 321, 960, 961, 2500])
def test_numbers_of_tensors(count):
    flat = _x((count * 37,), F32, 3)
    grads = list(flat.view(count, 37).unbind())       # off every vector boundary
    norm = _check_norm(step.grad_norm(grads), grads)
    out = torch.zeros_like(flat)
    step.clip_grads(grads, norm / 2, out=list(out.view(count, 37).unbind()))
    _check_clipped([out], [flat], 0.5)
    params = torch.ones_like(flat)
    step.sgd_step(list(params.view(count, 37).unbind()), grads, 1.0, max_norm=norm / 4)
    want = 1 - flat.double() / 4
    mo.close(params, want, mo.rounded(want, 9 * mo.E * flat.double().abs() + mo.E * want.abs(), F32))


def test_large_and_reproducible():
    grads = [_x((50304, 768), F32, 4, 1e-3), _x((9_000_011,), BF16, 5, 1e-3), _x((12_345_678,), F16, 6, 1e-3)]
    norm = _check_norm(step.grad_norm(grads), grads)
    assert all(torch.equal(step.grad_norm(grads), step.grad_norm(grads)) for _ in range(3))
    out = [torch.empty_like(g) for g in grads]
    step.clip_grads(grads, norm / 7, out=out)
    _check_clipped(out, grads, 1 / 7)
    step.clip_grads(grads, norm / 7)
    assert all(torch.equal(a, b) for a, b in zip(grads, out))


@pytest.mark.parametrize("size", [1e30, 1e20, 2.0 ** 60, 1.0, 2.0 ** -48, 1e-20, 1e-30, 1e-38, 1e-42])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_gradients_of_every_size(size, dtype):
    grads = [_x((3, 1000), F32, 7).mul(size).to(dtype), torch.zeros(5000, dtype=dtype, device="cuda"), _x((17,), F32, 8).mul(size).to(dtype)]
    norm = mo.norm(grads)
    got = step.grad_norm(grads)
    assert abs(float(got) - norm) <= mo.NORM_OFF * norm + 2.0 ** -149
    out = [torch.empty_like(g) for g in grads]
    step.clip_grads(grads, float(torch.tensor(norm / 2, dtype=F32)), out=out)
    if norm > 1e-36:
        _check_clipped(out, grads, float(torch.tensor(norm / 2, dtype=F32)) / norm)


def test_sizes_side_by_side():
    grads = [torch.full((9,), 3e38, device="cuda"), torch.full((4000,), 1e-3, device="cuda")]
    assert math.isinf(float(step.grad_norm(grads)))             # 9e38: more than the scalar holds
    out = [torch.empty_like(g) for g in grads]
    step.clip_grads(grads, 9.0, out=out)                        # the factor does not go by the scalar
    _check_clipped(out, grads, 9.0 / mo.norm(grads))
    tiny = [torch.full((16,), 1e-30, device="cuda"), torch.full((16,), 1.0, device="cuda")]
    _check_norm(step.grad_norm(tiny), tiny)


def test_infinities_and_nan():
    g = [_x((100,), F32, 9), _x((50,), BF16, 10)]
    g[1][7] = float("nan")
    before = [x.clone() for x in g]
    assert math.isnan(float(step.clip_grads(g, 1.0)))
    assert torch.equal(g[0], before[0]) and int(g[1].isnan().sum()) == 1 and torch.equal(g[1].nan_to_num(0.0), before[1].nan_to_num(0.0))
    g = [_x((100,), F32, 9), _x((50,), BF16, 10)]
    g[1][7] = float("inf")
    assert math.isinf(float(step.clip_grads(g, 1.0)))
    assert not bool(g[0].any()) and bool(g[1][7].isnan()) and not bool(g[1].nan_to_num(0.0).any())
    assert float(step.grad_norm([torch.zeros(3, device="cuda")])) == 0.0
    z = [torch.zeros(3, device="cuda")]
    assert float(step.clip_grads(z, 0.0)) == 0.0 and not bool(z[0].any())
    assert float(step.grad_norm([torch.empty(0, device="cuda")])) == 0.0


def test_strides():
    a, b, c = _x((40, 50), F32, 11), _x((40, 100), BF16, 12), _x((1, 50), F32, 13)
    grads = [a.t(), b[:, ::2], c.expand(40, -1), _x((3, 4, 5), F32, 14).permute(2, 0, 1)]
    norm = _check_norm(step.grad_norm(grads), grads)
    out = [torch.empty(g.shape, device="cuda") for g in grads]
    _check_norm(step.clip_grads(grads, norm / 2, out=out), grads)
    _check_clipped(out, grads, 0.5)
    out = [torch.empty_like(g, dtype=F32) for g in (grads[0], grads[3])]
    step.clip_grads([grads[0], grads[3]], 1e9, out=out)
    assert torch.equal(out[0], grads[0]) and torch.equal(out[1], grads[3])
    back = [torch.empty((50, 40), device="cuda").t().contiguous().t()]      # laid out the other way round
    step.clip_grads([grads[0]], 1e9, out=back)
    assert torch.equal(back[0], grads[0])
    mine = a.t().clone()
    step.clip_grads([mine], 0.5)
    _check_clipped([mine], [a.t()], 0.5 / mo.norm([a]))
    odd = torch.empty(70001, dtype=BF16, device="cuda")[1:]
    odd.copy_(_x((70000,), BF16, 15))
    _check_norm(step.grad_norm([odd]), [odd])
    to = torch.empty(70003, device="cuda")[3:]
    step.clip_grads([odd], 1.0, out=[to])
    _check_clipped([to], [odd], 1 / mo.norm([odd]))


def test_what_lies_beside_is_not_touched():
    room = torch.full((5 * 1000 + 64,), 9.0, device="cuda")
    grads = [_x((1000,), F32, 16 + i) for i in range(5)]
    step.clip_grads(grads, 1.0, out=[room[64 * (i > 2) + 1000 * i:][:1000] for i in range(5)])
    assert bool((room[3000:3064] == 9).all())


def test_another_stream_and_two_at_once():
    grads = [[_x((1_000_000,), F32, 30 + i)] for i in range(2)]
    want = [step.grad_norm(g) for g in grads]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = [None, None]
    for _ in range(10):
        for i in range(2):
            with torch.cuda.stream(streams[i]):
                got[i] = step.grad_norm(grads[i])
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_autograd_notices_what_is_written():
    w, x = torch.randn(64, device="cuda", requires_grad=True), torch.randn(64, device="cuda")
    for write in (lambda: step.clip_grads([x], 0.1), lambda: step.sgd_step([x], [torch.ones_like(x)], 0.1), lambda: step.clip_grads([torch.ones_like(x)], 0.1, out=[x])):
        y = (w * x).sum()
        write()
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            y.backward()
    inside = w * 2
    with pytest.raises(hb.HalosError):
        step.sgd_step([inside], [x], 0.1)
    with torch.no_grad():
        step.sgd_step([w], [x], 0.1)


@pytest.mark.parametrize("what", ["none", "cpu", "dtype", "not a tensor", "limit", "nan limit", "rate", "shapes", "fewer", "twice", "overlap", "onto another", "other type in place", "not dense", "broadcast"])
def test_refusals(what):
    g, kw, call = [_x((8,), F32, 40), _x((4, 6), F32, 41)], dict(max_norm=1.0), step.clip_grads
    if what == "none":
        g = []
    elif what == "cpu":
        g[1] = g[1].cpu()
    elif what == "dtype":
        g[1] = g[1].double()
    elif what == "not a tensor":
        g[1] = None
    elif what == "limit":
        kw = dict(max_norm=-1.0)
    elif what == "nan limit":
        kw = dict(max_norm=float("nan"))
    elif what == "rate":
        call, kw = (lambda g, **kw: step.sgd_step([x.clone() for x in g], g, **kw)), dict(rate=float("inf"))
    elif what == "shapes":
        kw["out"] = [g[0].clone(), g[1].t().contiguous()]
    elif what == "fewer":
        kw["out"] = [g[0].clone()]
    elif what == "twice":
        g = [g[0], g[0]]
    elif what == "overlap":
        room = torch.zeros(20, device="cuda")
        g = [g[0], g[0].clone()]
        kw["out"] = [room[:8], room[7:15]]
    elif what == "onto another":
        g = [g[0], g[0].clone()]
        kw["out"] = [g[1], torch.zeros(8, device="cuda")]
    elif what == "other type in place":
        kw["out"] = [g[0].view(torch.bfloat16)[:8], g[1].clone()]
    elif what == "not dense":
        g[1] = _x((4, 12), F32, 42)[:, ::2]
    elif what == "broadcast":
        g[1] = _x((1, 6), F32, 42).expand(4, -1)
    with pytest.raises(hb.HalosError) as e:
        call(g, **kw)
    assert e.value.status == hb.ERR_INVALID_ARG
