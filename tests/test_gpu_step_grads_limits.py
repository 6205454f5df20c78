"""Clipping and the step where the factor is smaller than 32 bits hold."""
from __future__ import annotations

import pytest
import torch

import step_more_oracle as mo
from paper_2506_04531_b200 import step

pytestmark = pytest.mark.gpu
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16


@pytest.mark.parametrize("limit", [1e-6, 1e-7, 1e-30, 2.0 ** -149])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n", [9, 8192, 40001])
def test_factors_below_32_bits(n, dtype, limit):
    """max_norm over the norm is subnormal, or nothing, in 32 bits; the clipped gradients are ordinary numbers, or as subnormal as max_norm is."""
    x = torch.randn(n, generator=torch.Generator(device="cuda").manual_seed(n), device="cuda").clamp(-3, 3)
    grads = [(x * 1e38).to(dtype), torch.full((9,), 3e38, device="cuda"), torch.ones(5, dtype=F16, device="cuda")]
    limit = float(torch.tensor(limit, dtype=F32))
    factor = limit / mo.norm(grads)
    assert factor < 2.0 ** -126
    for kinds in ((F32, F32, F32), (BF16, F32, F16)):
        out = [torch.full(g.shape, 7.0, dtype=t, device="cuda") for g, t in zip(grads, kinds)]
        step.clip_grads(grads, limit, out=out)
        for o, g in zip(out, grads):
            want = g.double() * factor
            mo.close(o, want, mo.rounded(want, 8 * mo.E * want.abs(), o.dtype))
        params = [torch.full(g.shape, limit, dtype=t, device="cuda") for g, t in zip(grads, kinds)]
        before = [p.clone() for p in params]
        step.sgd_step(params, grads, 0.25, max_norm=limit)
        for p, b, g in zip(params, before, grads):
            moved = 0.25 * factor * g.double()
            want = b.double() - moved
            mo.close(p, want, mo.rounded(want, 9 * mo.E * moved.abs() + mo.E * want.abs(), p.dtype))
    mine = [g.clone() for g in grads]
    step.clip_grads(mine, limit)
    for o, g in zip(mine, grads):
        want = g.double() * factor
        mo.close(o, want, mo.rounded(want, 8 * mo.E * want.abs(), o.dtype))


def test_a_factor_of_nothing():
    """rate 0 and max_norm 0 are held in 32 bits; a subnormal rate is, too."""
    g = torch.full((100,), 3e38, device="cuda")
    p = torch.ones(100, device="cuda")
    step.sgd_step([p], [g], 0.0)
    assert bool((p == 1).all())
    step.clip_grads([g], 0.0)
    assert not bool(g.any())
    g, rate = torch.full((100,), 3e38, device="cuda"), float(torch.tensor(1e-40, dtype=F32))
    step.sgd_step([p], [g], rate)
    want = 1 - rate * g.double()
    mo.close(p, want, mo.rounded(want, 2 * mo.E * want.abs(), F32))
