"""Gradients of the distillation from what its loss kept report what they do without it."""
import pytest
import torch

import paper_2607_08643_amd as bsq
from test_gpu_distill import Case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T", [40, 300, 1500])
@pytest.mark.parametrize("dt", [None, torch.bfloat16, torch.float32])
def test_words_past_the_vocabulary_are_reported_with_kept_too(T, dt, gpu):
    c = Case(gpu, T, 300, 64, 6, dead=0.2, seed=5)
    for bad in (False, True):
        for at in ((T - 1, 2), (3, 0)):
            ids = c.ids.clone()
            c.ids = c.ids.clone()
            if bad:
                c.ids[at[0]] = -1  # (also of a token that is left without words)
                c.ids[at] = 300
            loss, lse, kept = c.loss(keep=True)
            for k in (None, kept):
                err = torch.zeros(1, dtype=torch.int32, device=gpu)
                c.grad(lse, kept=k, head=dt is not None, dV=None if dt is None else torch.empty((300, 64), dtype=dt, device=gpu),
                       err=err)
                torch.cuda.synchronize()
                assert int(err.item()) == (bsq.DEVERR_BAD_SET if bad else 0)
            c.ids = ids
