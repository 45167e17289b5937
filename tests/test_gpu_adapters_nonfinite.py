"""Infinities and NaN in the weights or inputs of adapters reach what the formulas
say they reach, and nothing else: tokens without an adapter are the base alone,
sums over d_in have no terms past its end, gradients past an adapter's own rank
are 0."""
import pytest
import torch

import paper_2607_08643_amd as bsq
from parity_bounds import say
from test_gpu_adapters import Batch, _ids

pytestmark = pytest.mark.gpu

INF, NAN = float("inf"), float("nan")


def _spoil(q, a, value):
    """Adapter a's A and B hold `value` in places."""
    q.A[a, 0, 0], q.A[a, -1, -1] = value, value
    q.B[a, 0, 0], q.B[a, -1, -1] = value, -value


@pytest.mark.parametrize("value", [INF, NAN])
@pytest.mark.parametrize("y_dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("M,d_in,rank", [(40, 264, 16), (300, 264, 32), (1500, 96, 16), (1500, 77, 128)])
def test_a_spoiled_adapter_stays_alone(M, d_in, rank, y_dtype, value, gpu):
    """Whatever an adapter holds, tokens without one keep y0 and dx0, and other
    adapters' tokens and gradients their bits."""
    say(f"spoiled adapter M={M} d_in={d_in} rank={rank} {y_dtype} {value}")
    n = 3
    b = Batch(gpu, M, (96, 33), d_in, rank, n, _ids("mixed", M, n, 2), y_dtype=y_dtype)
    plan = bsq.bsq_adapters_plan(b.ids, n)
    g = torch.Generator().manual_seed(5)
    dy = [torch.randn((M, d), generator=g).bfloat16().to(gpu) for d in b.dims]
    base = torch.randn((M, d_in), generator=g).bfloat16().to(gpu)
    y, t = bsq.bsq_adapters_apply(plan, b.pools, b.X, b.base, keep=True)
    bare, _ = bsq.bsq_adapters_apply(plan, b.pools, b.X, None, y_dtype=y_dtype)
    dx, dA, dB = bsq.bsq_adapters_grad(plan, b.pools, b.X, t, dy, base=base)
    free, other = b.ids < 0, b.ids > 0
    assert free.any() and other.any()
    for q in b.pools:
        _spoil(q, 0, value)
    y2, t2 = bsq.bsq_adapters_apply(plan, b.pools, b.X, b.base, keep=True)
    bare2, _ = bsq.bsq_adapters_apply(plan, b.pools, b.X, None, y_dtype=y_dtype)
    dx2, dA2, dB2 = bsq.bsq_adapters_grad(plan, b.pools, b.X, t, dy, base=base)
    torch.cuda.synchronize()
    for p in range(2):
        assert torch.equal(y2[p][free], b.base[p][free]) and (bare2[p][free] == 0).all() and (t2[p][free] == 0).all()
        assert torch.equal(y2[p][other], y[p][other]) and torch.equal(bare2[p][other], bare[p][other])
        assert torch.equal(t2[p][other], t[p][other])
        assert torch.equal(dA2[p][1:], dA[p][1:]) and torch.equal(dB2[p][1:], dB[p][1:])
    assert torch.equal(dx2[free], base[free]) and torch.equal(dx2[other], dx[other])


@pytest.mark.parametrize("M", [40, 300, 1500])
@pytest.mark.parametrize("d_in", [8, 77, 264, 544, 1000])
def test_no_terms_past_the_end_of_d_in(M, d_in, gpu):
    """An infinite entry of A times x = 1 is an infinite t: nothing past d_in (where
    x has no values) is multiplied with it."""
    say(f"infinite A, M={M} d_in={d_in}")
    b = Batch(gpu, M, (40,), d_in, 16, 2, _ids("one", M, 2, 2))
    b.X[:, 0] = 1.0
    b.X[:, d_in - 1] = 1.0
    plan = bsq.bsq_adapters_plan(b.ids, 2)
    _, t = bsq.bsq_adapters_apply(plan, b.pools, b.X, None, keep=True)
    A = b.pools[0].A
    A[1, 2, 0], A[1, 7, 0], A[1, 9, d_in - 1] = INF, -INF, -INF
    _, u = bsq.bsq_adapters_apply(plan, b.pools, b.X, None, keep=True)
    torch.cuda.synchronize()
    want = t[0].clone()
    want[:, 2], want[:, 7], want[:, 9] = INF, -INF, -INF
    assert torch.equal(u[0], want)


@pytest.mark.parametrize("value", [INF, NAN])
@pytest.mark.parametrize("M", [40, 300, 5000])
def test_gradients_past_an_adapters_rank_are_zero(M, value, gpu):
    """Also where x or dy are not finite (0 times an infinity is no 0)."""
    say(f"gradients past the rank, M={M}, {value}")
    n, rank, own = 2, 20, [5, 0]
    b = Batch(gpu, M, (70,), 296, rank, n, _ids("mixed", M, n, 3), own)
    plan = bsq.bsq_adapters_plan(b.ids, n)
    _, t = bsq.bsq_adapters_apply(plan, b.pools, b.X, None, keep=True)
    dy = torch.randn((M, 70), generator=torch.Generator().manual_seed(1)).bfloat16().to(gpu)
    _, dA, dB = bsq.bsq_adapters_grad(plan, b.pools, b.X, t, [dy], want_dx=False)
    m = [int(b.tokens(a)[-1]) for a in range(n)]
    X2, dy2 = b.X.clone(), dy.clone()
    for k in m:
        X2[k, 3] = value
    _, dA2, dB2 = bsq.bsq_adapters_grad(plan, b.pools, X2, t, [dy], want_dx=False)
    for k in m:
        dy2[k, 11] = value
    before = ([torch.ones_like(dA[0])], [torch.ones_like(dB[0])])
    _, _, dB3 = bsq.bsq_adapters_grad(plan, b.pools, b.X, t, [dy2], want_dx=False)
    _, dA4, dB4 = bsq.bsq_adapters_grad(plan, b.pools, X2, t, [dy2], want_dx=False, grads=before, accumulate=True)
    torch.cuda.synchronize()
    for a, r in enumerate(own):
        assert (dA2[0][a, r:] == 0).all() and (dB3[0][a, :, r:] == 0).all()
        assert (dA4[0][a, r:] == 1).all() and (dB4[0][a, :, r:] == 1).all()
    keep = torch.arange(296, device=gpu) != 3
    assert torch.equal(dA2[0][:, :, keep], dA[0][:, :, keep]) and torch.equal(dB2[0], dB[0])
    assert not torch.isfinite(dA2[0][0, :5, 3]).any()
    keep = torch.arange(70, device=gpu) != 11
    assert torch.equal(dB3[0][:, keep], dB[0][:, keep]) and not torch.isfinite(dB3[0][0, 11, :5]).any()
