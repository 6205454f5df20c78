"""The embedding and its gradient against 64 bits: types, odd widths, tokens that come often, never or are none, strides, and writing onto what is there."""
from __future__ import annotations

import pytest
import torch
import torch.nn.functional as F

import step_more_oracle as mo
from paper_2506_04531_b200 import binding as hb, step

pytestmark = pytest.mark.gpu
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
PAIRS = [(F32, F32), (BF16, F32), (F16, F32), (BF16, BF16), (F16, F16), (F32, BF16), (F32, F16), (BF16, F16), (F16, BF16)]   # rows, table


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _x(shape, dtype, seed, scale=1.0):
    return (torch.randn(shape, generator=_gen(seed), device="cuda") * scale).to(dtype)


def _tokens(shape, vocab, seed, dtype=torch.int64):
    return torch.randint(0, vocab, shape, generator=_gen(seed), device="cuda").to(dtype)


@pytest.mark.parametrize("dtype,wtype", PAIRS)
@pytest.mark.parametrize("vocab,dim,shape,scale", [(1, 1, (1,), 1.0), (7, 3, (5,), 2.5), (50, 8, (3, 11), 1.0), (1000, 97, (4, 130), 0.37), (513, 64, (2, 3, 50), 8.0), (70, 768, (2, 257), 27.7),
                                                   (300, 1028, (150,), 1.0), (40, 2050, (70,), 1.0)])
def test_against_64_bits(dtype, wtype, vocab, dim, shape, scale):
    weight, tokens = _x((vocab, dim), wtype, 1), _tokens(shape, vocab, 2, torch.int32 if dim % 2 else torch.int64)
    y = step.embedding_forward(weight, tokens, scale=scale, dtype=dtype)
    assert y.dtype == dtype
    mo.close(y, *mo.embedding(weight, tokens, scale, dtype))
    dout = _x((*shape, dim), dtype, 3)
    dw = step.embedding_backward(dout, tokens, vocab, scale=scale, dtype=wtype)
    assert dw.dtype == wtype and dw.shape == weight.shape
    mo.close(dw, *mo.embedding_backward(dout, tokens, vocab, scale, wtype))
    assert torch.equal(dw, step.embedding_backward(dout, tokens, vocab, scale=scale, dtype=wtype))


@pytest.mark.parametrize("tokens,vocab", [(1, 50304), (31, 5), (32, 33), (33, 600), (1024, 70000), (1025, 511), (1025, 512), (1025, 513), (5000, 300000), (8192, 700), (8193, 40), (16385, 9), (40000, 97), (65536, 3000), (65537, 3000), (200000, 2000), (3000, 2 ** 27 + 5)])
def test_many_tokens_and_large_vocabularies(tokens, vocab):
    """One pass of the sort to four; more tokens than one block of it takes."""
    dim = 12 if vocab < 2 ** 20 else 2
    t = _tokens((tokens,), vocab, 4)
    t[-1], t[0] = vocab - 1, 0
    dout = _x((tokens, dim), BF16, 5)
    dw = step.embedding_backward(dout, t, vocab, dtype=F32)
    if vocab < 2 ** 20:
        mo.close(dw, *mo.embedding_backward(dout, t, vocab, 1.0, F32))
    else:
        met, at = torch.unique(t, return_inverse=True)
        mo.close(dw[met], *mo.embedding_backward(dout, at, met.numel(), 1.0, F32))
        dw[met] = 0
        assert not bool(dw.any())


@pytest.mark.parametrize("dim", [5, 64, 1000])
@pytest.mark.parametrize("n", [32, 63, 64, 65, 5000, 20000])
def test_one_token_everywhere(n, dim):
    """Its sum goes through many chunks; beside it one that comes once, before or after."""
    for other in (0, 9):
        t = torch.full((n,), 4, device="cuda")
        t[n // 2] = other
        dout = _x((n, dim), F16, 6)
        dw = step.embedding_backward(dout, t, 11, dtype=F32)
        mo.close(dw, *mo.embedding_backward(dout, t, 11, 1.0, F32))
        assert torch.equal(dw[other], dout[n // 2].float())


def test_runs_of_every_length():
    """Tokens that come 1, 2, ... 130 times, so that runs begin and end everywhere in a chunk; sums of ones are exact."""
    t = torch.repeat_interleave(torch.arange(130, device="cuda"), torch.arange(1, 131, device="cuda"))
    t = t[torch.randperm(t.numel(), generator=_gen(7), device="cuda")]
    for dim in (1, 40, 300):
        dw = step.embedding_backward(torch.ones((t.numel(), dim), device="cuda", dtype=BF16), t, 140, dtype=F32)
        assert torch.equal(dw[:130], torch.arange(1, 131, device="cuda", dtype=F32)[:, None].expand(-1, dim)) and not bool(dw[130:].any())


@pytest.mark.parametrize("wide", [True, False])
def test_tokens_that_are_none(wide):
    weight = _x((10, 24), F32, 8)
    t = torch.tensor([3, -1, 10, 9, 2 ** 31 - 1, -2 ** 31, 0] + ([2 ** 40 + 3, -2 ** 62] if wide else []), dtype=torch.int64 if wide else torch.int32, device="cuda")
    mo.close(step.embedding_forward(weight, t), *mo.embedding(weight, t, 1.0, F32))
    dout = _x((t.numel(), 24), F32, 9)
    mo.close(step.embedding_backward(dout, t, 10), *mo.embedding_backward(dout, t, 10, 1.0, F32))
    dout[1] = float("nan")
    assert not bool(step.embedding_backward(dout, t, 10).isnan().any())
    assert not bool(step.embedding_backward(dout, torch.full_like(t, -1), 10).any())


def test_what_rows_hold_stays_in_them():
    weight, t = _x((6, 40), BF16, 10), torch.tensor([0, 5, 5, 2, 3], device="cuda")
    weight[2, 3], weight[3] = float("nan"), float("inf")
    mo.close(step.embedding_forward(weight, t), *mo.embedding(weight, t, 1.0, BF16))
    dout = _x((5, 40), BF16, 11)
    dout[1, 7], dout[3] = float("nan"), float("-inf")
    mo.close(step.embedding_backward(dout, t, 6, dtype=F32), *mo.embedding_backward(dout, t, 6, 1.0, F32))


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_nothing_to_do(dtype):
    weight, none = _x((6, 8), dtype, 12), torch.empty((2, 0), dtype=torch.int64, device="cuda")
    assert step.embedding_forward(weight, none).shape == (2, 0, 8)
    out = torch.full((6, 8), 3.0, dtype=dtype, device="cuda")
    assert not bool(step.embedding_backward(torch.empty((2, 0, 8), dtype=dtype, device="cuda"), none, 6, out=out.clone()).any())
    assert torch.equal(step.embedding_backward(torch.empty((2, 0, 8), dtype=dtype, device="cuda"), none, 6, out=out, accumulate=True), torch.full_like(out, 3.0))
    assert step.embedding_forward(weight, torch.tensor(3, device="cuda")).shape == (8,)
    one = step.embedding_backward(torch.ones(8, dtype=dtype, device="cuda"), torch.tensor(3, device="cuda"), 6)
    assert float(one.double().sum()) == 8 and bool((one[3] == 1).all())


@pytest.mark.parametrize("dtype,wtype", [(BF16, F32), (F32, F32), (F16, F16)])
@pytest.mark.parametrize("dim", [33, 256])
def test_onto_what_is_there(dtype, wtype, dim):
    """Rows that no token names keep their bits, NaN included, and what lies between rows is not touched."""
    vocab, n = 50, 700
    room = _x((vocab, dim + 7), wtype, 13)
    room[40] = float("nan")
    before, t = room.clone(), _tokens((n,), 37, 14)
    dout = _x((n, dim), dtype, 15)
    got = step.embedding_backward(dout, t, vocab, scale=0.5, out=room[:, :dim], accumulate=True)
    assert got.data_ptr() == room.data_ptr()
    want, bound = mo.embedding_backward(dout, t, vocab, 0.5, wtype, before[:, :dim])
    mo.close(got, want, bound)
    named = torch.unique(t)
    rest = torch.ones(vocab, dtype=torch.bool, device="cuda")
    rest[named] = False
    same = lambda a, b: torch.equal(a.view(torch.int16 if a.element_size() == 2 else torch.int32), b.view(torch.int16 if a.element_size() == 2 else torch.int32))  # noqa: E731
    assert same(room[rest].contiguous(), before[rest].contiguous()) and same(room[:, dim:].contiguous(), before[:, dim:].contiguous())
    step.embedding_backward(dout, t, vocab, scale=0.5, out=room[:, :dim])
    mo.close(room[:, :dim], *mo.embedding_backward(dout, t, vocab, 0.5, wtype))
    assert same(room[:, dim:].contiguous(), before[:, dim:].contiguous())


@pytest.mark.parametrize("dtype,wtype", [(BF16, F32), (F32, F32), (F16, F16), (F32, BF16)])
@pytest.mark.parametrize("n", [1, 2, 31, 33, 255, 256, 257])
@pytest.mark.parametrize("how", ["apart", "one", "half", "none"])
def test_few_onto_what_is_there(dtype, wtype, n, how):
    """Every place another token, one token everywhere, one at every other place among others that are none, and none at all; a column more than whole warps take, rows apart."""
    vocab, dim = 400, 289
    room = _x((vocab, dim + 3), wtype, 60)
    room[399] = float("nan")
    t = torch.randperm(399, generator=_gen(61), device="cuda")[:n]
    if how != "apart":
        t = {"one": torch.full_like(t, 7), "half": torch.where(torch.arange(n, device="cuda") % 2 == 0, 7, torch.where(t % 3 == 0, -t - 1, t)), "none": t + vocab}[how]
    wide = _x((n, 2 * dim), dtype, 62)
    dout, before = wide[:, dim:], room.clone()
    if how == "half":
        dout[t < 0] = float("nan")       # no row's
    got = step.embedding_backward(dout, t, vocab, scale=0.5, out=room[:, :dim], accumulate=True)
    ok = (t >= 0) & (t < vocab)
    want, bound = mo.embedding_backward(dout[ok], t[ok], vocab, 0.5, wtype, before[:, :dim])
    mo.close(got[:399], want[:399], bound[:399])
    bits = torch.int16 if room.element_size() == 2 else torch.int32
    rest = torch.ones(vocab, dtype=torch.bool, device="cuda")
    rest[t[ok]] = False
    assert torch.equal(room[rest].view(bits), before[rest].view(bits)) and torch.equal(room[:, dim:].contiguous().view(bits), before[:, dim:].contiguous().view(bits))
    again = before.clone()
    step.embedding_backward(dout, t, vocab, scale=0.5, out=again[:, :dim], accumulate=True)
    assert torch.equal(again.view(bits), room.view(bits))


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_strides(dtype):
    wide = _x((90, 3, 40), dtype, 16)
    weight, t = wide[:, 1], _tokens((8, 30), 90, 17)
    assert torch.equal(step.embedding_forward(weight, t), step.embedding_forward(weight.contiguous(), t))
    assert torch.equal(step.embedding_forward(weight, t[:, 1:-1]), step.embedding_forward(weight.contiguous(), t[:, 1:-1].contiguous()))
    odd = torch.empty(90 * 40 + 1, dtype=dtype, device="cuda")[1:].view(90, 40)
    odd.copy_(weight)
    assert torch.equal(step.embedding_forward(odd, t), step.embedding_forward(weight.contiguous(), t))
    every = _x((8, 30, 2, 40), dtype, 18)
    plain = step.embedding_backward(every[:, :, 0].contiguous(), t, 90, dtype=F32)
    assert torch.equal(step.embedding_backward(every[:, :, 0], t, 90, dtype=F32), plain)
    assert torch.equal(step.embedding_backward(every.permute(0, 3, 2, 1)[:, :, 0].contiguous().permute(0, 2, 1), t, 90, dtype=F32), plain)
    assert torch.equal(step.embedding_backward(every[:, :1, 0].expand(-1, 30, -1), t, 90), step.embedding_backward(every[:, :1, 0].expand(-1, 30, -1).contiguous(), t, 90))
    off = torch.empty(every[:, :, 0].numel() + 1, dtype=dtype, device="cuda")[1:].view(8, 30, 40)
    off.copy_(every[:, :, 0])
    assert torch.equal(step.embedding_backward(off, t, 90, dtype=F32), plain)


def test_offsets_beyond_32_bits():
    vocab, dim = 600_000, 4096
    weight = torch.zeros((vocab, dim), dtype=F16, device="cuda")
    weight[-1], weight[vocab // 2] = 3.0, 2.0
    t = torch.tensor([vocab - 1, vocab // 2, 5, vocab - 1], dtype=torch.int32, device="cuda")
    assert step.embedding_forward(weight, t)[:, -1].tolist() == [3.0, 2.0, 0.0, 3.0]
    del weight
    dw = step.embedding_backward(torch.ones((4, dim), dtype=F16, device="cuda"), t, vocab)
    assert bool((dw[-1] == 2).all()) and bool((dw[vocab // 2] == 1).all()) and bool((dw[5] == 1).all()) and float(dw.sum(1, dtype=F32).sum()) == 4 * dim


def test_gradient_and_second_derivative():
    weight, t = _x((20, 16), F32, 19).requires_grad_(), _tokens((3, 9), 20, 20)
    other = weight.detach().double().requires_grad_()
    c = _x((3, 9, 16), F32, 21)
    y, z = step.embedding(weight, t, scale=3.0), F.embedding(t, other) * 3.0
    a, = torch.autograd.grad((y.pow(3) * c).sum(), weight, create_graph=True)
    b, = torch.autograd.grad((z.pow(3) * c).sum(), other, create_graph=True)
    assert torch.allclose(a.double(), b, rtol=1e-5, atol=1e-3)
    a2, = torch.autograd.grad(a.pow(2).sum(), weight)
    b2, = torch.autograd.grad(b.pow(2).sum(), other)
    assert float((a2.double() - b2).abs().max()) <= 1e-5 * float(b2.abs().max())
    h = step.embedding(weight, t, dtype=BF16)
    h.float().sum().backward()
    assert h.dtype == BF16 and weight.grad.dtype == F32 and float(weight.grad.sum()) == t.numel() * 16
    # against differences: linear, so any step will do
    way = _x((20, 16), F32, 22)
    slope = ((step.embedding_forward(weight.detach() + way, t) - step.embedding_forward(weight.detach() - way, t)) * c).sum() / 2
    got = (step.embedding_backward(c, t, 20) * way).sum()
    assert abs(float(got - slope)) <= 1e-4 * float((c.abs().sum()))


def test_another_stream():
    dout, t = _x((3000, 100), F32, 23), _tokens((3000,), 500, 24)
    want = step.embedding_backward(dout, t, 500)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        got = step.embedding_backward(dout, t, 500)
    side.synchronize()
    assert torch.equal(got, want)


@pytest.mark.parametrize("what", ["cpu", "table", "dtype", "weight", "strided", "tokens", "tokens cpu", "no columns", "no rows"])
def test_refusals_forward(what):
    weight, t, kw = _x((5, 8), F32, 25), torch.zeros(3, dtype=torch.int64, device="cuda"), {}
    if what == "cpu":
        weight = weight.cpu()
    elif what == "table":
        weight = weight[0]
    elif what == "dtype":
        kw = dict(dtype=torch.float64)
    elif what == "weight":
        weight = weight.double()
    elif what == "strided":
        weight = weight[:, ::2]
    elif what == "tokens":
        t = t.short()
    elif what == "tokens cpu":
        t = t.cpu()
    elif what == "no columns":
        weight = weight[:, :0]
    elif what == "no rows":
        weight = weight[:0]
    with pytest.raises(hb.HalosError) as e:
        step.embedding_forward(weight, t, **kw)
    assert e.value.status == hb.ERR_INVALID_ARG


@pytest.mark.parametrize("what", ["cpu", "shape", "dtype", "out shape", "out type", "out strided", "out broadcast", "accumulate", "vocab", "graph"])
def test_refusals_backward(what):
    dout, t, vocab, kw = _x((3, 8), F32, 26), torch.zeros(3, dtype=torch.int64, device="cuda"), 5, {}
    if what == "cpu":
        dout = dout.cpu()
    elif what == "shape":
        dout = dout[:2]
    elif what == "dtype":
        kw = dict(dtype=torch.float64)
    elif what == "out shape":
        kw = dict(out=torch.zeros(5, 7, device="cuda"))
    elif what == "out type":
        kw = dict(out=torch.zeros(5, 8, device="cuda"), dtype=BF16)
    elif what == "out strided":
        kw = dict(out=torch.zeros(5, 16, device="cuda")[:, ::2])
    elif what == "out broadcast":
        kw = dict(out=torch.zeros(1, 8, device="cuda").expand(5, -1), accumulate=True)
    elif what == "accumulate":
        kw = dict(accumulate=True)
    elif what == "vocab":
        vocab = 0
    elif what == "graph":
        kw = dict(out=torch.zeros(5, 8, device="cuda", requires_grad=True) * 1)
    with pytest.raises(hb.HalosError) as e:
        step.embedding_backward(dout, t, vocab, **kw)
    assert e.value.status == hb.ERR_INVALID_ARG
