"""Gradients whose norm fits 64 bits but not 32: the norm is reported as an
infinity, the gradients are clipped all the same."""
import math

import pytest
import torch

import paper_2607_08643_amd as bsq
from parity_bounds import say

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("max_norm", [1e38, 3.0, 1e-3])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_a_norm_past_the_range_of_32_bits(dtype, max_norm, gpu):
    """coef, in 32 bits, is off by 2^-24 of itself or, where it is below 2^-126, by half
    of 2^-149; out has that error, its own rounding of 2^-24 (bf16: 2^-8), and both
    once more for good measure."""
    say(f"clip {dtype} max {max_norm}")
    ts = [torch.full((5000,), 3e38, device=gpu).to(dtype), torch.full((3, 100), -1e38, device=gpu).to(dtype),
          torch.full((7,), 2.0, device=gpu).to(dtype)]
    norm = math.sqrt(sum(float(t.double().square().sum()) for t in ts))
    assert 3.5e38 < norm < 1e41
    coef = max_norm / (norm + 1e-6)
    off = max(2.0 ** -24 * coef, 2.0 ** -150)
    err = torch.zeros(1, dtype=torch.int32, device=gpu)
    outs = [torch.empty_like(t) for t in ts]
    stats = bsq.bsq_grad_clip(bsq.GradPlan(ts, outs), max_norm, err=err)
    alone = bsq.bsq_grad_norm(bsq.GradPlan(ts), max_norm)
    torch.cuda.synchronize()
    assert math.isinf(float(stats[0])) and torch.equal(alone, stats) and int(err.item()) == 0
    assert abs(float(stats[1]) - coef) <= 2 * off
    for t, o in zip(ts, outs):
        want = coef * t.double()
        bar = 2 * off * t.double().abs() + 2 * (2.0 ** -24 if dtype == torch.float32 else 2.0 ** -8) * want.abs() + 2.0 ** -133
        assert ((o.double() - want).abs() <= bar).all()
