"""The distillation loss and its gradient against the 64-bit form: types, odd vocabularies, strides, absent and doubled entries, ignored rows,
logits at the type's limits, and gradients against differences."""
from __future__ import annotations

import math

import pytest
import torch

import step_oracle as so
from paper_2506_04531_b200 import binding as hb, step

pytestmark = pytest.mark.gpu

DTYPES = [torch.float32, torch.bfloat16, torch.float16]


def _case(n, V, k, dtype, seed=0, spare=0, absent=True):
    g = torch.Generator(device="cuda").manual_seed(seed)
    z = (torch.randn((n, V + spare), generator=g, device="cuda") * 3).to(dtype)[:, :V]
    labels = torch.randint(0, V, (n,), generator=g, device="cuda")
    idx = torch.stack([torch.randperm(V, generator=g, device="cuda")[:k] for _ in range(n)]) if n else torch.zeros((0, k), dtype=torch.int64, device="cuda")
    t = (torch.randn((n, k), generator=g, device="cuda") * 2 + 5).to(dtype)
    if absent and n > 2:
        labels[1] = -100
        idx[2] = -1
        idx[:, k // 2:][torch.rand((n, k - k // 2), generator=g, device="cuda") < 0.3] = -1
    scale = 4096.0 if dtype == torch.float16 else 1.0
    return z, labels, idx, t, torch.rand(n, generator=g, device="cuda") * scale


def _within(got, want, bound, what):
    off = (got.double() - want).abs()
    assert bool(torch.isfinite(got).all()), what
    assert bool((off <= bound).all()), (what, float((off - bound).max()))


def _check(z, labels, idx, t, dloss, **how):
    how = {"temperature": 1.0, "mix": 0.5, "ignore_index": -100, **how}
    want = so.distill(z, labels, idx, t, dloss, **how)
    loss, stats = step.distill_forward(z, labels, idx, t, **how)
    _within(loss, want["loss"], want["loss_bound"], "loss")
    _within(stats, want["stats"], want["stats_bound"], "stats")
    dz = step.distill_backward(dloss, z, stats, labels, idx, t, **how)
    _within(dz, want["dz"], want["dz_bound"], "backward")
    loss2, dz2 = step.distill_loss_and_grad(z, labels, idx, t, dloss, **how)
    _within(loss2, want["loss"], want["loss_bound"], "loss of both")
    _within(dz2, want["dz"], want["dz_bound"], "gradient of both")
    own = z.clone(memory_format=torch.preserve_format) if z.is_contiguous() else z
    step.distill_loss_and_grad(own, labels, idx, t, dloss, out=own, **how)     # over the logits themselves
    assert torch.equal(own, dz2)
    return loss, dz


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("temperature", [1.0, 1.5, 2.0, 4.0, 0.5])
@pytest.mark.parametrize("n,V,k", [(1, 1, 1), (3, 2, 1), (5, 37, 8), (7, 1000, 20), (4, 4097, 64), (3, 50304, 64), (2, 70001, 100)])
def test_against_64_bits(n, V, k, temperature, dtype):
    _check(*_case(n, V, k, dtype, seed=V), temperature=temperature)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("temperature", [1.0, 3.0])
@pytest.mark.parametrize("V,spare", [(130003, 0), (130003, 5), (60000, 0)])
def test_rows_that_shared_memory_does_not_hold(V, spare, temperature, dtype):
    z, labels, idx, t, dloss = _case(3, V, 40, dtype, spare=spare)
    _check(z, labels, idx, t, dloss, temperature=temperature)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("mix", [0.0, 1.0])
@pytest.mark.parametrize("temperature", [1.0, 2.0, 3.0])
def test_one_term_alone(temperature, mix, dtype):
    z, labels, idx, t, dloss = _case(6, 5003, 17, dtype)
    _check(z, labels, idx, t, dloss, mix=mix, temperature=temperature)
    _check(z.contiguous(), None, idx, t, dloss, mix=0.6, temperature=temperature)
    _check(z.contiguous(), labels, None, None, dloss, mix=0.6, temperature=temperature)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("spare", [1, 8, 13, 40])
def test_rows_with_room_between_them(spare, dtype):
    z, labels, idx, t, dloss = _case(9, 1003, 12, dtype, spare=spare)
    a = _check(z.clone(memory_format=torch.contiguous_format), labels, idx, t, dloss, temperature=2.0)
    z2 = _case(9, 1003, 12, dtype, spare=spare)[0]
    loss, stats = step.distill_forward(z2, labels, idx, t, temperature=2.0)
    assert bool(((loss - a[0]).abs() <= 1e-4).all())
    # into an output whose rows start elsewhere
    out = torch.full((9, 1010), 7.0, dtype=dtype, device="cuda")
    step.distill_backward(dloss, z2, stats, labels, idx, t, temperature=2.0, out=out[:, 3:1006])
    want = so.distill(z2, labels, idx, t, dloss, temperature=2.0, mix=0.5, ignore_index=-100)
    _within(out[:, 3:1006], want["dz"], want["dz_bound"], "dz")
    assert bool((out[:, :3] == 7).all()) and bool((out[:, 1006:] == 7).all())
    _check(z2, labels, idx, t, dloss, temperature=2.0)


@pytest.mark.parametrize("labels_dtype", [torch.int32, torch.int64])
@pytest.mark.parametrize("index_dtype", [torch.int32, torch.int64])
@pytest.mark.parametrize("teacher_dtype", DTYPES)
def test_types_of_labels_and_teacher(teacher_dtype, index_dtype, labels_dtype):
    z, labels, idx, t, dloss = _case(5, 600, 30, torch.bfloat16)
    _check(z, labels.to(labels_dtype), idx.to(index_dtype), t.to(teacher_dtype), dloss, temperature=2.0, ignore_index=-100)


def test_doubled_entries_count_twice_and_meet_the_label():
    z, labels, idx, t, dloss = _case(4, 300, 6, torch.float32, absent=False)
    idx[:, 3] = idx[:, 0]
    idx[:, 4] = labels
    _check(z, labels, idx, t, dloss, temperature=2.0)


def test_k_at_its_limit():
    _check(*_case(2, 3000, 1024, torch.float32), temperature=1.0)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("low", ["lowest", -math.inf])
@pytest.mark.parametrize("temperature", [1.0, 2.0, 1.5])
def test_logits_at_the_types_limits(temperature, low, dtype):
    """A vocabulary padded with the type's lowest value or with -infinity, a row with nothing but the lowest, and one large logit."""
    z, labels, idx, t, dloss = _case(6, 700, 9, dtype, absent=False)
    low = torch.finfo(dtype).min if low == "lowest" else low
    labels, idx = labels % 400, idx % 400
    z[:, 400:] = low
    z[3, 0] = 90.0
    if low != -math.inf:
        z[4] = low
    how = dict(temperature=temperature, mix=0.5, ignore_index=-100)
    loss, dz = step.distill_loss_and_grad(z, labels, idx, t, dloss, **how)
    keep = [0, 1, 2, 3, 5]
    want = so.distill(z[keep][:, :400], labels[keep], idx[keep], t[keep], dloss[keep], **how)
    _within(loss[keep], want["loss"], want["loss_bound"], "loss")
    _within(dz[keep][:, :400], want["dz"], want["dz_bound"], "dz")
    assert float(dz[keep][:, 400:].abs().sum()) == 0
    if low != -math.inf:                    # all alike: uniform
        flat = so.distill(torch.zeros_like(z[4:5]), labels[4:5], idx[4:5], t[4:5], dloss[4:5], **how)
        if dtype != torch.float16:          # log of the sum drowns in 3e38, and so does the loss; the gradient is that of T = 1 or NaN-free at least
            assert not bool(torch.isnan(dz[4]).any())
        else:
            assert bool(((loss[4:5].double() - flat["loss"]).abs() <= 0.2).all())


def test_ignored_rows_may_hold_anything_and_give_nothing():
    z, labels, idx, t, dloss = _case(4, 500, 8, torch.bfloat16, absent=False)
    labels[:] = torch.tensor([3, 7, 7, 5], device="cuda")
    z[1], z[2] = float("nan"), float("inf")
    loss, dz = step.distill_loss_and_grad(z, labels, idx, t, dloss, ignore_index=7)
    _, stats = step.distill_forward(z, labels, idx, t, ignore_index=7)
    dz2 = step.distill_backward(dloss, z, stats, labels, idx, t, ignore_index=7)
    assert loss[1:3].tolist() == [0, 0] and float(dz[1:3].abs().sum()) == float(dz2[1:3].abs().sum()) == 0
    assert bool(torch.isfinite(dz).all()) and bool(torch.isfinite(loss).all()) and float(loss[0]) > 0


def test_indices_outside_the_vocabulary_come_back_as_nan():
    z, labels, idx, t, dloss = _case(4, 500, 8, torch.float32, absent=False)
    labels[0], labels[1], idx[2, 3] = 500, -5, 500
    loss, dz = step.distill_loss_and_grad(z, labels, idx, t, dloss)
    assert torch.isnan(loss).tolist() == [True, True, True, False]
    assert bool(torch.isnan(dz[:3]).all()) and not bool(torch.isnan(dz[3]).any())


@pytest.mark.parametrize("temperature", [1.0, 2.0, 1.5])
def test_gradient_against_differences(temperature):
    z, labels, idx, t, _ = _case(5, 211, 10, torch.float32)
    leaf = z.clone().requires_grad_()
    w = torch.tensor([0.3, 1.0, -2.0, 0.7, 1.1], device="cuda")
    (step.distill_loss(leaf, labels, idx, t, temperature=temperature, mix=0.4) * w).sum().backward()
    how = dict(temperature=temperature, mix=0.4, ignore_index=-100)
    form = lambda x: float((so.distill(x.to(torch.float64), labels, idx, t, None, **how)["loss"] * w.double()).sum())  # noqa: E731
    so.U[torch.float64], so.TINY[torch.float64] = 0.0, 0.0
    want = so.distill(z, labels, idx, t, w, **how)
    way, h = torch.randn(z.shape, generator=torch.Generator(device="cuda").manual_seed(1), device="cuda").double(), 1e-5
    slope = (form(z.double() + h * way) - form(z.double() - h * way)) / (2 * h)
    assert abs(float((leaf.grad.double() * way).sum()) - slope) <= float((want["dz_bound"] * way.abs()).sum()) + 1e-6 * abs(slope)


def test_empty_and_other_stream_and_same_bits():
    z, labels, idx, t, dloss = _case(0, 100, 4, torch.float32)
    loss, dz = step.distill_loss_and_grad(z, labels, idx, t, dloss)
    assert loss.shape == (0,) and dz.shape == (0, 100)
    z, labels, idx, t, dloss = _case(300, 5000, 16, torch.bfloat16)
    want = step.distill_loss_and_grad(z, labels, idx, t, dloss, temperature=2.0)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        got = step.distill_loss_and_grad(z, labels, idx, t, dloss, temperature=2.0)
    side.synchronize()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


@pytest.mark.parametrize("what,status", [("temperature", hb.ERR_INVALID_ARG), ("mix", hb.ERR_INVALID_ARG), ("k", hb.ERR_UNSUPPORTED), ("dtype", hb.ERR_INVALID_ARG), ("cpu", hb.ERR_INVALID_ARG),
                                         ("labels", hb.ERR_INVALID_ARG), ("teacher", hb.ERR_INVALID_ARG), ("dloss", hb.ERR_INVALID_ARG), ("out", hb.ERR_INVALID_ARG), ("columns", hb.ERR_INVALID_ARG),
                                         ("overlap", hb.ERR_INVALID_ARG)])
def test_refusals(what, status):
    z, labels, idx, t, dloss = _case(3, 2000, 1025 if what == "k" else 4, torch.float32, absent=False)
    kw = {}
    if what == "temperature":
        kw = dict(temperature=0.0)
    elif what == "mix":
        kw = dict(mix=1.5)
    elif what == "dtype":
        z = z.double()
    elif what == "cpu":
        labels = labels.cpu()
    elif what == "labels":
        labels = labels[:2]
    elif what == "teacher":
        t = None
    elif what == "dloss":
        dloss = dloss.double()
    elif what == "out":
        kw = dict(out=torch.empty(3, 1999, device="cuda"))
    elif what == "columns":
        z = z[:, ::2]
    elif what == "overlap":
        kw = dict(out=torch.empty(2000, device="cuda").expand(3, -1))
    with pytest.raises(hb.HalosError) as e:
        step.distill_loss_and_grad(z, labels, idx, t, dloss, **kw)
    assert e.value.status == status
