"""Adapters at ranks whose blocks of 16 reach past the rank (33 to 48, 65 to
112), against the formulas in fp64, with the bars of the other adapter tests."""
import pytest
import torch

import paper_2607_08643_amd as bsq
from parity_bounds import say
from test_gpu_adapters import Batch, _check_apply, _check_grad, _ids

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rank", [33, 48, 65, 96, 112])
@pytest.mark.parametrize("M,d_in,n,own", [(70, 264, 1, False), (300, 77, 3, True), (1100, 512, 2, False)])
def test_ranks_between_the_blocks(rank, M, d_in, n, own, gpu):
    say(f"adapters rank={rank} M={M} d_in={d_in} n={n} own ranks={own}")
    ranks = [rank - (i % 3) * (rank // 2) for i in range(n)] if own else None
    b = Batch(gpu, M, (96, 40), d_in, rank, n, _ids("mixed", M, n, 4), ranks, seed=rank)
    plan = bsq.bsq_adapters_plan(b.ids, n)
    y, t = bsq.bsq_adapters_apply(plan, b.pools, b.X, b.base, keep=True)
    torch.cuda.synchronize()
    _check_apply(b, y, t, b.base)
    g = torch.Generator().manual_seed(8)
    dy = [torch.randn((M, d), generator=g).bfloat16().to(gpu) for d in b.dims]
    for dt in (torch.bfloat16, torch.float32):
        dx, dA, dB = bsq.bsq_adapters_grad(plan, b.pools, b.X, t, dy, dx_dtype=dt)
        torch.cuda.synchronize()
        _check_grad(b, t, dy, None, dx, dA, dB, dt)
