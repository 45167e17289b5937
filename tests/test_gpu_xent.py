"""Cross entropy from hidden states (bsq_xent_loss, bsq_xent_grad) against the
definition in fp64: z = H V^T, lse = log sum exp(z), loss = lse - z_target,
d = g (exp(z - lse) - onehot), dH = d V, dV = d^T H.

Bars. A logit is a sum of D exact products that rounds at least after every four
of them: dz <= gamma(D) sum |h v|, gamma(n) = (n / 4 + 16) 2^-24. lse changes by
at most the largest dz; the exponentials and their sums add 2^-18 (each 2^-21,
and the sum's own roundings, tile by tile) and the last logarithm and addition
2^-23 of |lse|. In the gradient d is off by |g| p (dz + 2^-18) and rounded to
bf16, an error uniform on half an ulp (at most 2^-8 |d|), whose sum over
independent terms exceeds 3.78 * 2^-8 * sqrt(sum of squares) with probability
under 1e-9; then the second product's gamma and the rounding of the result.
"""
import pytest
import torch

import paper_2607_08643_amd as bsq
from parity_bounds import SUBGAUSS, say

pytestmark = pytest.mark.gpu

U32 = 2.0 ** -24
U16 = 2.0 ** -8
IGNORE = -100


def gamma(n):
    return (n / 4 + 16) * U32


def _inputs(gpu, T, N, D, ignore=0.0, seed=1, pad=0, std=1.0):
    g = torch.Generator().manual_seed(seed)
    V = torch.randn((N, D), generator=g).mul(std / D ** 0.5).bfloat16()
    target = torch.randint(0, N, (T,), generator=g)
    lift = torch.rand((T, 1), generator=g) * 8
    H = (torch.randn((T, D), generator=g) + lift * V[target].float() * (1 / std)).bfloat16()
    target[torch.rand(T, generator=g) < ignore] = IGNORE

    def rows(t):
        buf = torch.full((t.shape[0], D + pad), float("nan"), dtype=torch.bfloat16, device=gpu)
        buf[:, :D] = t
        return buf[:, :D]
    return rows(H), rows(V), target.to(gpu)


def _exact(H, V, target):
    live = target >= 0
    h, v = H[live].double(), V.double()
    z = h @ v.T
    dz = gamma(H.shape[1]) * (h.abs() @ v.abs().T)
    lse = torch.logsumexp(z, 1)
    return live, h, v, z, dz, lse


def _check_loss(H, V, target, loss, lse):
    live, h, v, z, dz, want = _exact(H, V, target)
    t = target[live][:, None]
    want_loss = want - z.gather(1, t)[:, 0]
    tol = dz.amax(1) + 2.0 ** -18 + 2.0 ** -23 * want.abs() if live.any() else want
    for name, got, ref, bar in (("lse", lse, want, tol), ("loss", loss, want_loss, tol + dz.gather(1, t)[:, 0] if live.any() else tol)):
        assert (got[~live] == 0).all()
        err = (got[live].double() - ref).abs()
        say(f"  {name}: worst err/tol {float((err / bar).max()) if len(err) else 0:.4f}")
        assert (err <= bar).all(), name


SHAPES = [
    # T, N, D, ignored, row padding
    (1, 1, 8, 0.0, 0),
    (1, 5000, 256, 0.0, 0),
    (3, 255, 72, 0.0, 8),
    (16, 257, 64, 0.3, 0),
    (17, 1000, 1000, 0.0, 0),
    (33, 3001, 128, 0.5, 0),
    (64, 512, 40, 0.0, 24),
    (65, 777, 136, 0.0, 0),
    (128, 2050, 320, 0.2, 0),
    (129, 1030, 264, 0.0, 0),
    (300, 32003, 200, 0.4, 0),
    (513, 4100, 512, 0.9, 8),
    (50, 300, 64, 1.0, 0),
    (1030, 1500, 96, 0.0, 0),
]


@pytest.mark.parametrize("T,N,D,ignore,pad", SHAPES)
def test_loss_matches_definition(T, N, D, ignore, pad, gpu):
    say(f"xent loss T={T} N={N} D={D} ignore={ignore}")
    H, V, target = _inputs(gpu, T, N, D, ignore, pad=pad)
    loss, lse = bsq.bsq_xent_loss(H, V, target)
    torch.cuda.synchronize()
    _check_loss(H, V, target, loss, lse)


def _check_grad(H, V, target, lse, g, dH, dV, dv_dtype=torch.bfloat16, before=None):
    live, h, v, z, dz, _ = _exact(H, V, target)
    gl = g[live].double()[:, None]
    p = (z - lse[live].double()[:, None]).exp()
    d = p.clone()
    if live.any():
        d[torch.arange(len(d), device=d.device), target[live]] -= 1
    d, ed = gl * d, gl.abs() * (p * (dz.expm1() + 2.0 ** -18) + U32 * d.abs())
    want = d @ v
    tol = SUBGAUSS * U16 * (d.square() @ v.square()).sqrt() + (ed + gamma(V.shape[0]) * d.abs()) @ v.abs() + U16 * want.abs() + 1e-30
    assert (dH[~live] == 0).all()
    err = (dH[live].double() - want).abs()
    say(f"  dH: worst err/tol {float((err / tol).max()) if err.numel() else 0:.3f}")
    assert (err <= tol * 1.01).all()
    if dV is None:
        return
    want = d.T @ h
    tol = SUBGAUSS * U16 * (d.square().T @ h.square()).sqrt() + (ed + gamma(len(d)) * d.abs()).T @ h.abs() + 1e-30
    if before is not None:
        want = want + before.double()
        tol += U32 * want.abs()
    tol += (U16 if dv_dtype == torch.bfloat16 else U32) * want.abs()
    err = (dV.double() - want).abs()
    say(f"  dV: worst err/tol {float((err / tol).max()):.3f}")
    assert (err <= tol * 1.01).all()


def _weights(T, seed, gpu):
    return (torch.rand(T, generator=torch.Generator().manual_seed(seed)) * 2 - 0.5).to(gpu)


@pytest.mark.parametrize("T,N,D,ignore,pad", SHAPES)
def test_gradients_match_definition(T, N, D, ignore, pad, gpu):
    say(f"xent grad T={T} N={N} D={D} ignore={ignore}")
    H, V, target = _inputs(gpu, T, N, D, ignore, seed=2, pad=pad)
    g = _weights(T, 5, gpu)
    _, lse = bsq.bsq_xent_loss(H, V, target)
    g[target < 0] = float("nan")  # not read
    dH, dV = bsq.bsq_xent_grad(H, V, target, lse, g)
    torch.cuda.synchronize()
    _check_grad(H, V, target, lse, g, dH, dV)
    frozen, none = bsq.bsq_xent_grad(H, V, target, lse, g, head=False)
    assert none is None and torch.equal(frozen, dH)
    # added to 32-bit sums, and to bf16 ones
    for dt in (torch.float32, torch.bfloat16):
        before = torch.randn((N, D), generator=torch.Generator().manual_seed(3)).to(dt).to(gpu)
        acc = before.clone()
        bsq.bsq_xent_grad(H, V, target, lse, g, dV=acc, accumulate=True)
        torch.cuda.synchronize()
        _check_grad(H, V, target, lse, g, dH, acc, dt, before)


def test_pieces_of_the_vocabulary_add_up(gpu):
    """Enough tokens and words that d does not fit one piece: the last is short."""
    T, N, D = 4000, 40003, 64
    say(f"xent pieces T={T} N={N} D={D}")
    H, V, target = _inputs(gpu, T, N, D, 0.1, seed=7)
    loss, lse = bsq.bsq_xent_loss(H, V, target)
    g = _weights(T, 6, gpu)
    dH, dV = bsq.bsq_xent_grad(H, V, target, lse, g)
    torch.cuda.synchronize()
    _check_loss(H, V, target, loss, lse)
    _check_grad(H, V, target, lse, g, dH, dV)


def test_gradients_match_differences(gpu):
    """Central differences of sum g loss, in fp64, along random directions."""
    T, N, D = 70, 600, 64
    H, V, target = _inputs(gpu, T, N, D, 0.2, seed=4)
    g = _weights(T, 8, gpu)
    _, lse = bsq.bsq_xent_loss(H, V, target)
    dH, dV = bsq.bsq_xent_grad(H, V, target, lse, g)
    live = target >= 0
    h0, v0, t, w = H[live].double(), V.double(), target[live][:, None], g[live].double()

    def value(h, v):
        z = h @ v.T
        return float((w * (torch.logsumexp(z, 1) - z.gather(1, t)[:, 0])).sum())

    eps = 1e-5  # differences off by eps^2 and 1e-16 / eps of a value: under 1e-9
    for seed in range(4):
        gen = torch.Generator().manual_seed(seed)
        eh, ev = (torch.randn(s, generator=gen, dtype=torch.float64).to(gpu) for s in (h0.shape, v0.shape))
        for got, e, f in ((dH[live], eh, lambda s: value(h0 + s * eh, v0)), (dV, ev, lambda s: value(h0, v0 + s * ev))):
            diff = (f(eps) - f(-eps)) / (2 * eps)
            along = float((got.double() * e).sum())
            # two roundings of 2^-8 per element, independent
            bar = SUBGAUSS * 2 * U16 * float((got.double() * e).square().sum().sqrt()) * 2 + 1e-6
            say(f"  difference {diff:.6f}, gradient {along:.6f}, bar {bar:.6f}")
            assert abs(diff - along) <= bar


def test_tokens_without_a_loss_may_hold_anything(gpu):
    T, N, D = 200, 900, 128
    H, V, target = _inputs(gpu, T, N, D, 0.3, seed=3)
    g = _weights(T, 2, gpu)
    loss, lse = bsq.bsq_xent_loss(H, V, target)
    want = bsq.bsq_xent_grad(H, V, target, lse, g)
    dead = target < 0
    H2, g2, lse2 = H.clone(), g.clone(), lse.clone()
    H2[dead], g2[dead], lse2[dead] = float("nan"), float("inf"), float("nan")
    loss2, lse3 = bsq.bsq_xent_loss(H2, V, target)
    got = bsq.bsq_xent_grad(H2, V, target, lse2, g2)
    torch.cuda.synchronize()
    assert torch.equal(loss, loss2) and torch.equal(lse, lse3)
    assert torch.equal(want[0], got[0]) and torch.equal(want[1], got[1])


def test_a_target_past_the_vocabulary_is_reported(gpu):
    H, V, target = _inputs(gpu, 40, 300, 64)
    target[7], target[9] = 300, 1 << 40
    err = torch.zeros(1, dtype=torch.int32, device=gpu)
    loss, lse = bsq.bsq_xent_loss(H, V, target, err=err)
    torch.cuda.synchronize()
    assert int(err.item()) == bsq.DEVERR_BAD_SET
    masked = torch.where(target >= 300, -1, target)
    _check_loss(H, V, masked, loss, lse)
    err.zero_()
    bsq.bsq_xent_loss(H, V, masked, err=err)
    torch.cuda.synchronize()
    assert int(err.item()) == 0


def test_logits_of_any_size(gpu):
    """Logits of thousands and rows of -inf words: the largest is subtracted tile by tile."""
    T, N, D = 20, 1300, 64
    H, V, target = _inputs(gpu, T, N, D, seed=9)
    H[:10] *= 512
    V[:, 0] = 0
    V[300:600, 0] = float("-inf")  # whole tiles' words with z = -inf where h > 0
    H[:, 0] = 1
    target = torch.where((target >= 300) & (target < 600), 7, target)
    loss, lse = bsq.bsq_xent_loss(H, V, target)
    torch.cuda.synchronize()
    keep = torch.cat([torch.arange(300), torch.arange(600, N)]).to(gpu)
    place = torch.full((N,), -1, device=gpu)
    place[keep] = torch.arange(len(keep), device=gpu)
    _check_loss(H, V[keep].contiguous(), place[target], loss, lse)


def test_no_tokens(gpu):
    H, V = torch.empty((0, 64), dtype=torch.bfloat16, device=gpu), torch.randn((100, 64), device=gpu).bfloat16()
    none = torch.empty(0, dtype=torch.int64, device=gpu)
    loss, lse = bsq.bsq_xent_loss(H, V, none)
    assert loss.shape == (0,) and lse.shape == (0,)
    dV = torch.ones_like(V)
    dH, _ = bsq.bsq_xent_grad(H, V, none, lse, lse, dV=dV)
    torch.cuda.synchronize()
    assert dH.shape == (0, 64) and (dV == 0).all()


def test_results_repeat_and_a_captured_step_replays(gpu):
    T, N, D = 270, 2000, 200
    H, V, target = _inputs(gpu, T, N, D, 0.2, seed=6)
    g = _weights(T, 1, gpu)

    def step(stream=None):
        loss, lse = bsq.bsq_xent_loss(H, V, target, stream=stream)
        dH, dV = bsq.bsq_xent_grad(H, V, target, lse, g, stream=stream)
        return [loss, lse, dH, dV]

    want = step()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    other = step(side)
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = step()
    for _ in range(3):
        for q in held:
            q.fill_(5.0)
        graph.replay()
        torch.cuda.synchronize()
        again = step()
        torch.cuda.synchronize()
        for q, w, x in zip(held, want, again):
            assert torch.equal(q, w) and torch.equal(x, w)
    for q, w in zip(other, want):
        assert torch.equal(q, w)


def test_rows_past_32_bit_offsets(gpu):
    N, ld, T, D = 300, 1 << 23, 40, 64
    H, V, target = _inputs(gpu, T, N, D, seed=5)
    g = _weights(T, 4, gpu)
    big = torch.empty(N * ld, dtype=torch.bfloat16, device=gpu).view(N, ld)
    W, dW = big[:, :D], big[:, 128:128 + D]
    W.copy_(V)
    loss, lse = bsq.bsq_xent_loss(H, V, target)
    loss2, lse2 = bsq.bsq_xent_loss(H, W, target)
    dH, dV = bsq.bsq_xent_grad(H, V, target, lse, g)
    dH2, _ = bsq.bsq_xent_grad(H, W, target, lse, g, dV=dW)
    torch.cuda.synchronize()
    assert torch.equal(loss, loss2) and torch.equal(lse, lse2) and torch.equal(dH, dH2) and torch.equal(dV, dW)
