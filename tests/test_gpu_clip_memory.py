"""A plan of gradients is of the memory that they had: it stays theirs while the
plan is there, whatever becomes of the tensor objects."""
import gc

import pytest
import torch

import paper_2607_08643_amd as bsq

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("with_outs", [False, True])
def test_a_plan_keeps_the_memory_of_its_tensors(with_outs, gpu):
    n = 3 << 20  # (a size of its own among the allocator's blocks)
    grads = [torch.full((n,), 3.0, device=gpu), torch.full((n,), 4.0, device=gpu)]
    outs = [torch.zeros(n, device=gpu) for _ in grads] if with_outs else None
    held = {t.data_ptr() for t in grads + (outs or [])}
    plan = bsq.GradPlan(grads, outs)
    for t in grads + (outs or []):
        t.data = torch.zeros(1, device=gpu)
    gc.collect()
    others = [torch.full((n,), 9.0, device=gpu) for _ in range(8)]
    assert not held & {t.data_ptr() for t in others}
    stats = bsq.bsq_grad_clip(plan, 1.0)
    torch.cuda.synchronize()
    assert abs(float(stats[0]) - 5.0 * n ** 0.5) <= 2.0 ** -23 * 5.0 * n ** 0.5
    assert all((t == 9.0).all() for t in others)
