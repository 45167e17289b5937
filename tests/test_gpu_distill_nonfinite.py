"""Gradients of the distillation of tokens whose logits have no softmax."""
import pytest
import torch

from test_gpu_distill import Case

pytestmark = pytest.mark.gpu

INF = float("inf")


@pytest.mark.parametrize("T", [40, 300])
def test_a_student_without_a_probability_is_no_number(T, gpu):
    """Tokens whose logits are all -inf have no softmax: their gradients are NaN with what was kept as
    without it, those of the others are as they were."""
    c = Case(gpu, T, 600, 64, 7, absent=0.0, seed=6)
    c.H[:, 0] = 0
    c.V[:, 0] = 1
    _, lse, kept = c.loss(keep=True)
    want = [c.grad(lse, kept=k, head=False)[0] for k in (None, kept)]
    c.H = c.H.clone()
    c.H[5, 0] = -INF
    _, lse, kept = c.loss(keep=True)
    other = torch.arange(T, device=gpu) != 5
    for k, w in zip((None, kept), want):
        dH, dV = c.grad(lse, kept=k)
        torch.cuda.synchronize()
        assert float(lse[5]) == -INF or bool(lse[5].isnan())
        assert dH[5].isnan().all() and torch.equal(dH[other], w[other])
        assert dV.isnan().all()
