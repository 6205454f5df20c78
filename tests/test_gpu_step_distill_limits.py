"""The distillation loss where its inputs are not what they should be: a teacher that has diverged, indices outside the vocabulary."""
from __future__ import annotations

import math

import pytest
import torch

from paper_2506_04531_b200 import step

pytestmark = pytest.mark.gpu

DTYPES = [torch.float32, torch.bfloat16, torch.float16]
# a row to a warp; rows in shared memory, by small and by large CTAs; rows that shared memory does not hold
VOCABS = [500, 9001, 40003, 130003]


def _case(n, V, k, dtype, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    z = (torch.randn((n, V), generator=g, device="cuda") * 3).to(dtype)
    labels = torch.randint(0, V, (n,), generator=g, device="cuda")
    idx = torch.stack([torch.randperm(V, generator=g, device="cuda")[:k] for _ in range(n)])
    t = (torch.randn((n, k), generator=g, device="cuda") * 2 + 5).to(dtype)
    return z, labels, idx, t, torch.rand(n, generator=g, device="cuda") + 0.5


def _both_ways(z, labels, idx, t, dloss, **how):
    """(loss, gradient) in one pass and in two."""
    loss, stats = step.distill_forward(z, labels, idx, t, **how)
    return [step.distill_loss_and_grad(z, labels, idx, t, dloss, **how), (loss, step.distill_backward(dloss, z, stats, labels, idx, t, **how))]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("V", VOCABS)
@pytest.mark.parametrize("value", [math.nan, math.inf])
@pytest.mark.parametrize("labelled", [True, False])
def test_a_teacher_that_is_no_number_shows_in_loss_and_gradient(labelled, value, V, dtype):
    z, labels, idx, t, dloss = _case(4, V, 40, dtype)
    labels = labels if labelled else None
    clean = _both_ways(z, labels, idx, t, dloss, temperature=1.5)
    t = t.clone()
    t[1, 33] = value
    t[2, :] = value
    for (loss, dz), (loss0, dz0) in zip(_both_ways(z, labels, idx, t, dloss, temperature=1.5), clean):
        assert torch.isnan(loss).tolist() == [False, True, True, False]
        assert bool(torch.isnan(dz[1, idx[1]]).all()) and bool(torch.isnan(dz[2, idx[2]]).all())
        assert torch.equal(loss[[0, 3]], loss0[[0, 3]]) and torch.equal(dz[[0, 3]], dz0[[0, 3]])


@pytest.mark.parametrize("V", VOCABS)
def test_an_ignored_row_hides_its_teacher(V):
    z, labels, idx, t, dloss = _case(3, V, 8, torch.float32)
    labels[1], t[1] = -100, math.nan
    for loss, dz in _both_ways(z, labels, idx, t, dloss):
        assert float(loss[1]) == 0 and float(dz[1].abs().sum()) == 0 and bool(torch.isfinite(loss).all()) and bool(torch.isfinite(dz).all())


@pytest.mark.parametrize("V", VOCABS)
def test_entries_of_minus_infinity_are_as_if_they_were_not_there(V):
    z, labels, idx, t, dloss = _case(3, V, 8, torch.float32)
    there = t.clone()
    there[0, 4:], there[1] = -math.inf, -math.inf
    absent = idx.clone()
    absent[0, 4:], absent[1] = -1, -1
    for (loss, dz), (loss2, dz2) in zip(_both_ways(z, labels, idx, there, dloss), _both_ways(z, labels, absent, t, dloss)):
        assert torch.equal(loss, loss2) and bool(torch.isfinite(dz).all())
        assert bool(((dz - dz2).abs() <= 2.0 ** -20 * dz2.abs() + 1e-30).all())


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("V", VOCABS)
@pytest.mark.parametrize("others", [True, False])
def test_an_index_outside_the_vocabulary_gives_nan_without_labels_too(others, V, dtype):
    z, _, idx, t, dloss = _case(3, V, 8, dtype)
    if not others:                                  # nothing valid beside it
        idx[1] = -1
    idx[1, 5] = V
    for loss, dz in _both_ways(z, None, idx, t, dloss, temperature=2.0):
        assert torch.isnan(loss).tolist() == [False, True, False]
        assert bool(torch.isnan(dz[1]).all()) and bool(torch.isfinite(dz[[0, 2]]).all())
