"""Global gradient norm and clipping (bsq_grad_norm, bsq_grad_clip) against fp64:
norm = sqrt(sum g^2), coef = min(1, max_norm / (norm + 1e-6)), out = coef g.

Bars: the squares are exact in fp64 and their fp64 sum is off by under 2^-28 of
itself at these sizes, so norm and coef carry their rounding to fp32 alone: 2^-24
(2^-23 taken). out = coef g in fp32 has both (2^-22), and a bf16 result its own
2^-8.
"""
import math

import pytest
import torch

import paper_2607_08643_amd as bsq
from parity_bounds import say

pytestmark = pytest.mark.gpu


def _tensors(gpu, sizes, seed=1, offset=0):
    g = torch.Generator().manual_seed(seed)
    out = []
    for i, n in enumerate(sizes):
        dt = torch.bfloat16 if i % 3 == 1 else torch.float32
        buf = torch.full((n + offset + 8,), float("nan"), dtype=dt, device=gpu)
        buf[offset:offset + n] = torch.randn(n, generator=g).to(gpu) * 10.0 ** (i % 5 - 2)
        out.append(buf[offset:offset + n])
    return out


def _norm(ts):
    return math.sqrt(sum(float(t.double().square().sum()) for t in ts))


def _check(ts, outs, stats, max_norm):
    norm = _norm(ts)
    coef = min(1.0, max_norm / (norm + 1e-6))
    got = stats.double().tolist()
    assert abs(got[0] - norm) <= 2.0 ** -23 * norm and abs(got[1] - coef) <= 2.0 ** -23 * coef
    for t, o in zip(ts, outs):
        if coef == 1.0:
            assert torch.equal(t, o)
            continue
        bar = 2.0 ** -22 + (2.0 ** -8 if t.dtype == torch.bfloat16 else 0.0)
        want = t.double() * coef
        assert ((o.double() - want).abs() <= bar * want.abs()).all()


SIZES = [
    [1], [7, 0, 3], [16384], [16385, 16383, 1], [100000, 3, 50001, 16384 * 3], [5] * 200, [0], [40_000_001, 64],
]


@pytest.mark.parametrize("sizes", SIZES, ids=lambda s: f"{len(s)}x{max(s)}")
@pytest.mark.parametrize("offset", [0, 1, 4])
@pytest.mark.parametrize("max_norm", [1.0, 1e9])
def test_norm_and_clip_match_formula(sizes, offset, max_norm, gpu):
    say(f"clip {len(sizes)} tensors up to {max(sizes)}, offset {offset}, max {max_norm}")
    ts = _tensors(gpu, sizes, offset=offset)
    outs = [torch.full_like(t, 3.0) for t in ts]
    plan = bsq.GradPlan(ts, outs)
    before = [t.clone() for t in ts]
    stats = bsq.bsq_grad_clip(plan, max_norm)
    torch.cuda.synchronize()
    _check(before, outs, stats, max_norm)
    assert all(torch.equal(t, b) for t, b in zip(ts, before))
    inplace = bsq.GradPlan(ts)
    assert torch.equal(bsq.bsq_grad_norm(inplace, max_norm), stats)
    assert torch.equal(bsq.bsq_grad_clip(inplace, max_norm), stats)
    torch.cuda.synchronize()
    assert all(torch.equal(t, o) for t, o in zip(ts, outs))


def test_norms_past_the_range_of_32_bit_squares(gpu):
    for scale in (1e25, 1e-30):
        ts = [torch.full((5000,), scale, device=gpu), torch.full((300,), -scale, device=gpu).bfloat16()]
        stats = bsq.bsq_grad_norm(bsq.GradPlan(ts), 1.0)
        norm = _norm(ts)
        assert abs(float(stats[0]) - norm) <= 2.0 ** -23 * norm


@pytest.mark.parametrize("value", [float("nan"), float("inf"), float("-inf")])
@pytest.mark.parametrize("which", [0, 1])
def test_a_norm_that_is_not_finite_clips_nothing_and_is_reported(value, which, gpu):
    ts = _tensors(gpu, [70000, 1000])
    err = torch.zeros(1, dtype=torch.int32, device=gpu)
    plan = bsq.GradPlan(ts)
    bsq.bsq_grad_norm(plan, 1.0, err=err)
    torch.cuda.synchronize()
    assert int(err.item()) == 0
    ts[which][500] = value
    before = [t.clone() for t in ts]
    stats = bsq.bsq_grad_clip(plan, 1.0, err=err)
    torch.cuda.synchronize()
    assert int(err.item()) == bsq.DEVERR_NONFINITE
    assert not math.isfinite(float(stats[0])) and float(stats[1]) == 1.0
    assert all(torch.equal(t.view(torch.int16), b.view(torch.int16)) for t, b in zip(ts, before))


def test_a_tensor_past_32_bit_offsets(gpu):
    n = (1 << 31) + 12345
    t = torch.zeros(n, dtype=torch.bfloat16, device=gpu)
    t[0], t[n - 1], t[n // 2] = 3.0, 4.0, 12.0
    stats = bsq.bsq_grad_clip(bsq.GradPlan([t]), 6.5)
    torch.cuda.synchronize()
    assert abs(float(stats[0]) - 13.0) < 1e-5
    assert [float(t[i]) for i in (0, n // 2, n - 1)] == [1.5, 6.0, 2.0]
    assert int((t != 0).sum()) == 3


def test_results_repeat_and_a_captured_call_replays(gpu):
    ts = _tensors(gpu, [300000, 77, 50000])
    outs = [torch.empty_like(t) for t in ts]
    plan = bsq.GradPlan(ts, outs)
    stats = torch.empty(2, device=gpu)
    bsq.bsq_grad_clip(plan, 1.0, stats=stats)
    want, wo = stats.clone(), [o.clone() for o in outs]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        bsq.bsq_grad_clip(plan, 1.0, stats=stats)
    for _ in range(3):
        for o in outs:
            o.zero_()
        stats.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(stats, want) and all(torch.equal(o, w) for o, w in zip(outs, wo))
        assert torch.equal(bsq.bsq_grad_clip(plan, 1.0), want)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = bsq.bsq_grad_clip(plan, 1.0, stream=side)
    side.synchronize()
    assert torch.equal(got, want)
