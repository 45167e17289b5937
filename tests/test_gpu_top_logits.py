"""The largest logits of a vocabulary's rows (bsq_top_logits) against a stable
sort, exactly, and the log of the sum of exponentials against 64 bits.

Bar of lse: an exponential's argument is rounded three times (2^-24 each, of an
argument whose mean under the softmax is at most log N < 22), the exponential 2^-22,
each sum of a lane's words and the joins some 2^9 2^-24 at most: 2^-14 for rows past
2^17 words, 2^-18 below (a lane sums under 2^5 words there); the last logarithm, product
and addition 2^-22 of |lse| and of |scale z|.
"""
import pytest
import torch

import paper_2607_08643_amd as bsq
from parity_bounds import say

pytestmark = pytest.mark.gpu

INF, NAN = float("inf"), float("nan")


def _sorted(Z, K):
    """Ids and values by the definition."""
    z = Z.float().cpu()
    z = torch.where(z.isnan(), -INF, z)
    top, ids = z.sort(dim=1, descending=True, stable=True)  # -0 and +0 are equal
    top, ids = top[:, :K], ids[:, :K]
    ids = torch.where(top > -INF, ids, -1).int()
    top = torch.where(top > -INF, top, -INF)
    pad = K - ids.shape[1]
    return torch.nn.functional.pad(ids, (0, pad), value=-1), torch.nn.functional.pad(top, (0, pad), value=-INF)


def _check(Z, K, scale=1.0, got=None):
    ids, top, lse = bsq.bsq_top_logits(Z, K, scale=scale) if got is None else got
    torch.cuda.synchronize()
    want_ids, want_top = _sorted(Z, K)
    assert torch.equal(ids.cpu(), want_ids)
    assert torch.equal(top.cpu(), want_top)
    x = Z.double().cpu() * scale
    want = torch.logsumexp(x, 1)
    fine = want.isfinite()
    peak = x.amax(1).abs()
    bar = (2.0 ** -14 if Z.shape[1] > 1 << 17 else 2.0 ** -18) + 2.0 ** -22 * (want.abs() + peak)
    err = (lse.cpu().double() - want).abs()
    say(f"  lse: worst err/bar {float((err / bar)[fine].max()) if fine.any() else 0:.4f}")
    assert (err <= bar)[fine].all()
    odd = lse.cpu().double()[~fine]
    assert torch.equal(odd.isnan(), want[~fine].isnan()) and torch.equal(odd[~odd.isnan()], want[~fine][~odd.isnan()])


def _rows(gpu, T, N, dtype, seed=1, pad=0, lead=0):
    g = torch.Generator().manual_seed(seed)
    buf = torch.full((T, lead + N + pad), NAN, dtype=dtype, device=gpu)
    z = buf[:, lead:lead + N]
    z.copy_(torch.randn((T, N), generator=g) * 3)
    return z


SHAPES = [
    # T, N, K, pad, lead
    (1, 1, 1, 0, 0),
    (1, 1, 256, 0, 0),
    (3, 7, 4, 0, 0),
    (5, 100, 256, 3, 1),
    (4, 511, 64, 0, 0),
    (4, 513, 1, 0, 0),
    (2, 1000, 200, 0, 0),
    (33, 4095, 17, 2, 3),
    (2, 4097, 256, 0, 0),
    (9, 8192, 8, 0, 0),
    (1, 8193, 64, 0, 0),
    (70, 32003, 50, 0, 5),
    (2, 151936, 64, 0, 0),
    (1, 300001, 255, 0, 0),
    (2100, 300, 9, 0, 0),
]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("T,N,K,pad,lead", SHAPES)
def test_matches_a_stable_sort(T, N, K, pad, lead, dtype, gpu):
    say(f"top T={T} N={N} K={K} {dtype}")
    _check(_rows(gpu, T, N, dtype, pad=pad, lead=lead), K, scale=0.7)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("N", [900, 20000, 151936])
@pytest.mark.parametrize("K", [1, 64, 256])
def test_rows_that_are_hard_to_cut(N, K, dtype, gpu):
    """Equal values, few values, rising and falling order, masks, zeros of both signs."""
    say(f"top N={N} K={K} {dtype}")
    g = torch.Generator().manual_seed(5)
    z = torch.zeros((12, N))
    z[0] = 1.5
    z[1] = torch.arange(N) / 64
    z[2] = -torch.arange(N) / 64
    z[3] = torch.randint(0, 3, (N,), generator=g).float()
    z[4] = -INF
    z[5] = torch.where(torch.rand(N, generator=g) < 0.99, -INF, torch.randn(N, generator=g))
    z[6] = torch.where(torch.rand(N, generator=g) < 0.5, 0.0, -0.0)
    z[7] = -INF
    z[7, N // 2] = -3.0
    z[8] = torch.finfo(dtype).min
    z[9, N - 1] = 1e-40
    z[10] = torch.randn(N, generator=g) * 1e4
    z[11] = (torch.arange(N) // 100).float()
    _check(z.to(dtype).to(gpu), K)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_nan_and_infinities(dtype, gpu):
    Z = _rows(gpu, 6, 9000, dtype, seed=3)
    Z[0, 17] = NAN
    Z[1, 40:8500] = NAN
    Z[2, 8999] = INF
    Z[3, [5, 4000, 8998]] = INF
    Z[4] = NAN
    Z[5, ::2] = -INF
    _check(Z, 40, scale=0.5)


@pytest.mark.parametrize("scale", [2.0 ** -64, 1e-3, 30.0, 2.0 ** 64])
def test_scales_of_any_size(scale, gpu):
    _check(_rows(gpu, 5, 9001, torch.float32, seed=6), 12, scale=scale)


def test_no_lse_and_given_outputs(gpu):
    Z = _rows(gpu, 20, 3001, torch.bfloat16)
    ids, top, lse = bsq.bsq_top_logits(Z, 10, want_lse=False)
    assert lse is None
    outs = (torch.zeros_like(ids), torch.zeros_like(top), torch.zeros(20, device=gpu))
    got = bsq.bsq_top_logits(Z, 10, ids=outs[0], top=outs[1], lse=outs[2])
    torch.cuda.synchronize()
    assert all(a is b for a, b in zip(got, outs)) and torch.equal(ids, got[0]) and torch.equal(top, got[1])
    _check(Z, 10, got=got)


def test_no_rows(gpu):
    ids, top, lse = bsq.bsq_top_logits(torch.empty((0, 50), device=gpu), 3)
    assert ids.shape == (0, 3) and top.shape == (0, 3) and lse.shape == (0,)


def test_rows_past_32_bit_offsets(gpu):
    ld = (1 << 31) + 5
    Z = torch.empty(2 * ld + 5000, dtype=torch.bfloat16, device=gpu).as_strided((3, 5000), (ld, 1))
    Z.copy_(_rows(gpu, 3, 5000, torch.bfloat16, seed=8))
    _check(Z, 30)


def test_another_stream_and_a_captured_call(gpu):
    Z = _rows(gpu, 40, 30011, torch.bfloat16, seed=4)
    other = _rows(gpu, 40, 30011, torch.bfloat16, seed=9)
    want = bsq.bsq_top_logits(Z, 33)
    want_other = bsq.bsq_top_logits(other, 33)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = bsq.bsq_top_logits(Z, 33, stream=side)
    side.synchronize()
    for a, b in zip(got, want):
        assert torch.equal(a, b)
    held_in = Z.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = bsq.bsq_top_logits(held_in, 33)
    for src, ref in ((Z, want), (other, want_other), (Z, want)):
        held_in.copy_(src)
        graph.replay()
        torch.cuda.synchronize()
        again = bsq.bsq_top_logits(src, 33)
        torch.cuda.synchronize()
        for a, b, c in zip(held, ref, again):
            assert torch.equal(a, b) and torch.equal(c, b)
