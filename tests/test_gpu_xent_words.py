"""Cross entropy with words of -inf (masked out of the vocabulary) at any depth,
head gradients in 32 bits, and vocabularies past what one launch holds."""
import math

import pytest
import torch

import paper_2607_08643_amd as bsq
from parity_bounds import say
from test_gpu_xent import U32, _check_grad, _check_loss, _exact, _inputs, _weights, gamma

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


@pytest.mark.parametrize("T,N,D,ignore", [(1, 5000, 256, 0.0), (33, 200, 64, 0.5), (65, 777, 136, 0.0), (300, 3001, 200, 0.4),
                                          (1030, 1500, 96, 0.0), (4000, 40003, 64, 0.1)])
def test_head_gradients_in_32_bits(T, N, D, ignore, gpu):
    """d enters a 32-bit dV as two bf16 parts: the first leaves at most 2^-9 of a
    value, the second at most 2^-9 of that. Bar: 2^-17 of every |d|, d's own error
    as in the other tests, the product's gamma over both parts, the result's
    rounding."""
    say(f"xent dV fp32 T={T} N={N} D={D}")
    H, V, target = _inputs(gpu, T, N, D, ignore, seed=12)
    g = _weights(T, 5, gpu)
    _, lse = bsq.bsq_xent_loss(H, V, target)
    live, h, v, z, dz, _ = _exact(H, V, target)
    gl = g[live].double()[:, None]
    p = (z - lse[live].double()[:, None]).exp()
    d = p.clone()
    d[torch.arange(len(d), device=d.device), target[live]] -= 1
    d, ed = gl * d, gl.abs() * (p * (dz.expm1() + 2.0 ** -18) + U32 * d.abs())
    want = d.T @ h
    bar = (ed + (2.0 ** -17 + gamma(2 * len(d))) * d.abs()).T @ h.abs() + 1e-30
    for before in (None, torch.randn((N, D), generator=torch.Generator().manual_seed(3)).to(gpu)):
        dV = torch.full((N, D), 3.0, device=gpu) if before is None else before.clone()
        dH, _ = bsq.bsq_xent_grad(H, V, target, lse, g, dV=dV, accumulate=before is not None)
        torch.cuda.synchronize()
        ref = want if before is None else want + before.double()
        err = (dV.double() - ref).abs()
        tol = bar + 2 * U32 * ref.abs()
        say(f"  dV: worst err/tol {float((err / tol).max()):.3f}")
        assert (err <= tol).all()
        _check_grad(H, V, target, lse, g, dH, None)


def test_a_vocabulary_of_more_tiles_than_a_launch_holds(gpu):
    """2^23 + 8 tiles of 512 threads are 2^32 work items and more. Logits are 0 but for
    four words, so lse is known: log(N - 4 + sum exp z), off by the additions of a
    token's 2^20 tiles (each of 32 threads 2^15 of them, one rounding each: 2^-9)."""
    T, N, D = 1024, (1 << 28) + 5, 8
    say(f"xent loss T={T} N={N} D={D}")
    words = [5, N // 2, N - 300, N - 1]
    value = [19.0, 18.5, 20.0, 18.0]
    V = torch.zeros((N, D), dtype=torch.bfloat16, device=gpu)
    for w, x in zip(words, value):
        V[w, 3] = x
    H = torch.zeros((T, D), dtype=torch.bfloat16, device=gpu)
    H[:, 3] = 1.0
    H[1::2, 3] = 0.5
    target = torch.tensor([words[i % 4] if i % 8 < 6 else 1000 + i for i in range(T)], device=gpu)
    loss, lse = bsq.bsq_xent_loss(H, V, target)
    torch.cuda.synchronize()
    for i in range(T):
        s = 0.5 if i % 2 else 1.0
        want = math.log(N - 4 + sum(math.exp(s * x) for x in value))
        z = s * value[i % 4] if i % 8 < 6 else 0.0
        assert abs(float(lse[i]) - want) <= 2.0 ** -9 + 2.0 ** -18, i
        assert abs(float(loss[i]) - (want - z)) <= 2.0 ** -9 + 2.0 ** -18, i
