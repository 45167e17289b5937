"""Cross entropy with words of -inf (masked out of the vocabulary) at any depth."""
import pytest
import torch

import paper_2607_08643_amd as bsq
from parity_bounds import say
from test_gpu_xent import _check_grad, _check_loss, _inputs, _weights

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("D", [8, 64, 72, 96, 1000])
@pytest.mark.parametrize("T", [1, 20, 64, 200, 1100])
def test_words_of_minus_infinity(T, D, gpu):
    """z = -inf has probability 0: loss, gradients and the other words' rows are
    those of the vocabulary without these words. (dH's column 0 is a sum of 0
    times -inf there, so it says nothing.)"""
    say(f"xent -inf words T={T} D={D}")
    N = 1300
    H, V, target = _inputs(gpu, T, N, D, seed=9)
    V[:, 0] = 0
    V[300:600, 0] = float("-inf")
    H[:, 0] = 1
    target = torch.where((target >= 300) & (target < 600), 7, target)
    loss, lse = bsq.bsq_xent_loss(H, V, target)
    keep = torch.cat([torch.arange(300), torch.arange(600, N)]).to(gpu)
    place = torch.full((N,), -1, device=gpu)
    place[keep] = torch.arange(len(keep), device=gpu)
    W, word = V[keep].contiguous(), place[target]
    torch.cuda.synchronize()
    _check_loss(H, W, word, loss, lse)
    g = _weights(T, 3, gpu)
    dH, dV = bsq.bsq_xent_grad(H, V, target, lse, g)
    torch.cuda.synchronize()
    assert (dV[300:600] == 0).all()
    dH[:, 0] = 0
    _check_grad(H, W, word, lse, g, dH, dV[keep])
