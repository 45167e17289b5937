"""Distillation from a teacher's top logits (bsq_distill_loss, bsq_distill_grad)
against the definition in fp64: p_k = exp(s a_k - norm), z = s H V^T, q = softmax(z),
loss = sum_k p_k (log p_k - log q_id_k), d = g s (P q - p), dH = d V, dV = d^T H.

Bars. A logit is a sum of D exact products that rounds at least after every four of
them, times the scale: dz <= s gamma(D) sum |h v| + 2^-24 |z|. lse changes by at most the
largest dz; the exponentials and their sums add 2^-18, the result's rounding 2^-24 of
|lse|. The loss is off by sum p dz + P (lse's error), the roundings of p and P to 32
bits (2^-24 of p_k |z_k| and P |lse|) and its own. d is off by |g| s P q (dz + 2^-18) and five
roundings of 2^-24 of its two terms (and by 2^-11 of P q from kept exponentials, but for
the teacher's words), then rounded to bf16: an error uniform on half an ulp
(at most 2^-8 |d|), whose sum over independent terms exceeds 3.78 * 2^-8 * sqrt(sum of
squares) with probability under 1e-9; then the second product's gamma and the
rounding of the result. A dV of 32 bits, and up to 128 tokens all results, take d in
two bf16 parts: 2^-9 of 2^-9 of a value is left, at most 2^-17.
"""
import pytest
import torch

import paper_2607_08643_amd as bsq
from parity_bounds import SUBGAUSS, say

pytestmark = pytest.mark.gpu

U32 = 2.0 ** -24
U16 = 2.0 ** -8
INF, NAN = float("inf"), float("nan")


def gamma(n):
    return (n / 4 + 16) * U32


class Case:
    def __init__(self, gpu, T, N, D, K, dead=0.0, absent=0.2, norm=False, scale=0.75, seed=1, pad=0):
        g = torch.Generator().manual_seed(seed)
        V = torch.randn((N, D), generator=g).div(D ** 0.5).bfloat16()
        ids = torch.randint(0, N, (T, K), generator=g)
        border = [w for w in (0, 255, 256, 511, 512, N - 1) if w < N][:K]
        ids[0, :len(border)] = torch.tensor(border)
        lift = torch.rand((T, 1), generator=g) * 6
        H = (torch.randn((T, D), generator=g) + lift * V[ids[:, 0]].float()).bfloat16()
        ids[torch.rand((T, K), generator=g) < absent] = -1
        ids[torch.rand(T, generator=g) < dead] = -1
        top = torch.randn((T, K), generator=g) * 3 + 9
        top[:, 0] += 4
        there = ids >= 0
        a = torch.where(there, top.double() * scale, -INF)
        more = torch.rand(T, generator=g) * 0.3

        def rows(t):
            buf = torch.full((t.shape[0], D + pad), NAN, dtype=torch.bfloat16, device=gpu)
            buf[:, :D] = t
            return buf[:, :D]
        self.H, self.V = rows(H), rows(V)
        self.ids, self.top = ids.int().to(gpu), top.to(gpu)
        self.norm = (torch.logsumexp(a, 1) + more).float().to(gpu) if norm else None
        self.scale = scale
        self.g = (torch.rand(T, generator=g) * 2 - 0.5).to(gpu)
        self.live = there.any(1).to(gpu)

    def loss(self, **kw):
        return bsq.bsq_distill_loss(self.H, self.V, self.ids, self.top, norm=self.norm, scale=self.scale, **kw)

    def grad(self, lse, **kw):
        return bsq.bsq_distill_grad(self.H, self.V, self.ids, self.top, lse, self.g, norm=self.norm, scale=self.scale, **kw)

    def exact(self):
        """Of the live tokens: h, v, p, log p, z, dz."""
        i = self.live
        h, v, ids = self.H[i].double(), self.V.double(), self.ids[i].long()
        a = torch.where(ids >= 0, self.top[i].double() * self.scale, -INF)
        logp = torch.log_softmax(a, 1) if self.norm is None else a - self.norm[i].double()[:, None]
        z = self.scale * (h @ v.T)
        dz = self.scale * gamma(h.shape[1]) * (h.abs() @ v.abs().T) + U32 * z.abs()
        return h, v, ids.clamp_min(0), torch.where(ids >= 0, logp.exp(), 0.0), logp, z, dz


def _check_loss(c, loss, lse):
    torch.cuda.synchronize()
    h, v, at, p, logp, z, dz = c.exact()
    assert (loss[~c.live] == 0).all() and (lse[~c.live] == 0).all()
    if not c.live.any():
        return
    want = torch.logsumexp(z, 1)
    tol = dz.amax(1) + 2.0 ** -18 + U32 * want.abs()
    err = (lse[c.live].double() - want).abs()
    say(f"  lse: worst err/tol {float((err / tol).max()):.4f}")
    assert (err <= tol).all()
    zk, P = z.gather(1, at), p.sum(1)
    want_loss = torch.where(p > 0, p * (logp - zk), 0.0).sum(1) + P * want
    tol = (p * dz.gather(1, at)).sum(1) + P * tol + U32 * ((p * zk.abs()).sum(1) + P * want.abs() + want_loss.abs())
    err = (loss[c.live].double() - want_loss).abs()
    say(f"  loss: worst err/tol {float((err / tol).max()):.4f}")
    assert (err <= tol).all()


def _check_grad(c, lse, dH, dV, before=None, kept=False):
    torch.cuda.synchronize()
    h, v, at, p, logp, z, dz = c.exact()
    assert (dH[~c.live] == 0).all()
    gs = c.g[c.live].double()[:, None] * c.scale
    q = (z - lse[c.live].double()[:, None]).exp() * p.sum(1, keepdim=True)
    t = torch.zeros_like(q).scatter_add_(1, at, p)
    d = gs * (q - t)
    ed = gs.abs() * (q * (dz.expm1() + 2.0 ** -18) + 5 * U32 * (q + t))
    if kept:
        ed += torch.where(t > 0, 0.0, 2.0 ** -11 * d.abs())
    want = d @ v
    two = len(c.g) <= 128  # d in two bf16 parts
    tol = (ed + (2.0 ** -17 if two else 0) * d.abs() + gamma(2 * v.shape[0]) * d.abs()) @ v.abs() + U16 * want.abs() + 1e-30
    if not two:
        tol += SUBGAUSS * U16 * (d.square() @ v.square()).sqrt()
    err = (dH[c.live].double() - want).abs()
    say(f"  dH: worst err/tol {float((err / tol).max()) if err.numel() else 0:.3f}")
    assert (err <= tol * 1.01).all()
    if dV is None:
        return
    want = d.T @ h
    if dV.dtype == torch.bfloat16 and not two:
        tol = SUBGAUSS * U16 * (d.square().T @ h.square()).sqrt() + (ed + gamma(len(d)) * d.abs()).T @ h.abs() + 1e-30
    else:
        tol = (ed + (2.0 ** -17 + gamma(2 * len(d))) * d.abs()).T @ h.abs() + 1e-30
    if before is not None:
        want = want + before.double()
    tol += (U16 if dV.dtype == torch.bfloat16 else 2 * U32) * want.abs() + (0 if before is None else U32 * want.abs())
    err = (dV.double() - want).abs()
    say(f"  dV {dV.dtype}: worst err/tol {float((err / tol).max()):.3f}")
    assert (err <= tol * 1.01).all()


SHAPES = [
    # T, N, D, K, dead, absent, norm, pad
    (1, 1, 8, 1, 0.0, 0.0, False, 0),
    (1, 5000, 256, 64, 0.0, 0.0, True, 0),
    (3, 255, 72, 256, 0.0, 0.2, False, 8),
    (16, 257, 64, 5, 0.3, 0.2, True, 0),
    (17, 1000, 1000, 33, 0.0, 0.5, False, 0),
    (33, 3001, 128, 200, 0.5, 0.2, True, 0),
    (64, 512, 40, 2, 0.0, 0.4, False, 24),
    (65, 777, 136, 100, 0.0, 0.2, True, 0),
    (128, 2050, 320, 64, 0.2, 0.0, False, 0),
    (129, 1030, 264, 16, 0.0, 0.2, True, 0),
    (300, 32003, 200, 50, 0.4, 0.2, False, 0),
    (513, 4100, 512, 64, 0.9, 0.2, True, 8),
    (50, 300, 64, 7, 1.0, 0.2, False, 0),
    (1030, 1500, 96, 65, 0.1, 0.2, True, 0),
]


@pytest.mark.parametrize("T,N,D,K,dead,absent,norm,pad", SHAPES)
def test_loss_matches_definition(T, N, D, K, dead, absent, norm, pad, gpu):
    say(f"distill loss T={T} N={N} D={D} K={K}")
    c = Case(gpu, T, N, D, K, dead, absent, norm, pad=pad)
    loss, lse = c.loss()
    _check_loss(c, loss, lse)
    loss2, lse2, kept = c.loss(keep=True)
    torch.cuda.synchronize()
    assert torch.equal(loss, loss2) and torch.equal(lse, lse2)


@pytest.mark.parametrize("T,N,D,K,dead,absent,norm,pad", SHAPES)
def test_gradients_match_definition(T, N, D, K, dead, absent, norm, pad, gpu):
    say(f"distill grad T={T} N={N} D={D} K={K}")
    c = Case(gpu, T, N, D, K, dead, absent, norm, seed=2, pad=pad)
    c.g[~c.live] = NAN  # not read
    _, lse, kept = c.loss(keep=True)
    dH, dV = c.grad(lse)
    _check_grad(c, lse, dH, dV)
    near, far = c.grad(lse, kept=kept)
    _check_grad(c, lse, near, far, kept=True)
    frozen, none = c.grad(lse, kept=kept, head=False)
    assert none is None and torch.equal(frozen, near)
    frozen, none = c.grad(lse, head=False)
    assert none is None and torch.equal(frozen, dH)
    # added to 32-bit sums, and to bf16 ones
    for dt in (torch.float32, torch.bfloat16):
        before = torch.randn((N, D), generator=torch.Generator().manual_seed(3)).to(dt).to(gpu)
        for k in (None, kept):
            acc = before.clone()
            a, _ = c.grad(lse, kept=k, dV=acc, accumulate=True)
            exact = k is None or dt == torch.float32  # (a dV of 32 bits does not take what is kept)
            assert torch.equal(a, dH if exact else near)
            _check_grad(c, lse, a, acc, before, kept=not exact)


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32])
def test_pieces_of_the_vocabulary_add_up(dt, gpu):
    """Enough tokens and words that d does not fit one piece: the last is short."""
    T, N, D = 4000, 40003, 64
    c = Case(gpu, T, N, D, 40, 0.1, seed=7, norm=True)
    loss, lse, kept = c.loss(keep=True)
    _check_loss(c, loss, lse)
    out = [c.grad(lse, kept=k, dV=torch.empty((N, D), dtype=dt, device=gpu)) for k in (None, kept)]
    _check_grad(c, lse, *out[0])
    _check_grad(c, lse, *out[1], kept=dt == torch.bfloat16)


def test_gradients_match_differences(gpu):
    """Central differences of sum g loss, in fp64, along random directions."""
    c = Case(gpu, 70, 600, 64, 20, 0.2, seed=4)
    _, lse = c.loss()
    dH, dV = c.grad(lse)
    h0, v0, at, p, logp, _, _ = c.exact()
    w = c.g[c.live].double()

    def value(h, v):
        logq = torch.log_softmax(c.scale * (h @ v.T), 1)
        return float((w * torch.where(p > 0, p * (logp - logq.gather(1, at)), 0.0).sum(1)).sum())

    eps = 1e-5  # differences off by eps^2 and 1e-16 / eps of a value: under 1e-9
    for seed in range(4):
        gen = torch.Generator().manual_seed(seed)
        eh, ev = (torch.randn(s, generator=gen, dtype=torch.float64).to(gpu) for s in (h0.shape, v0.shape))
        for got, e, f in ((dH[c.live], eh, lambda s: value(h0 + s * eh, v0)), (dV, ev, lambda s: value(h0, v0 + s * ev))):
            diff = (f(eps) - f(-eps)) / (2 * eps)
            along = float((got.double() * e).sum())
            # two roundings of 2^-8 per element, independent
            bar = SUBGAUSS * 2 * U16 * float((got.double() * e).square().sum().sqrt()) * 2 + 1e-6
            say(f"  difference {diff:.6f}, gradient {along:.6f}, bar {bar:.6f}")
            assert abs(diff - along) <= bar


def test_words_in_any_order_and_twice(gpu):
    """The order of a token's words changes nothing; a word listed twice counts twice; absent ones not at all."""
    c = Case(gpu, 40, 900, 128, 30, seed=3)
    _, lse = c.loss()
    order = torch.argsort(torch.rand((40, 30), generator=torch.Generator().manual_seed(1)), 1).to(gpu)
    c.ids, c.top = c.ids.gather(1, order).contiguous(), c.top.gather(1, order).contiguous()
    for change in range(3):
        if change == 1:
            c.ids[:, 1::2] = c.ids[:, ::2]
        elif change == 2:
            c.ids[:] = c.ids[:, :1]
        c.live = (c.ids >= 0).any(1)
        loss, again = c.loss()
        _check_loss(c, loss, again)
        _check_grad(c, again, *c.grad(again))
        same = c.live  # (no sum of the student's depends on the words)
        assert torch.equal(lse[same], again[same])


def test_tokens_without_words_may_hold_anything(gpu):
    c = Case(gpu, 200, 900, 128, 12, 0.3, seed=3, norm=True)
    loss, lse = c.loss()
    want = c.grad(lse)
    dead = ~c.live
    c.H, lse3 = c.H.clone(), lse.clone()
    c.H[dead], c.g[dead], lse3[dead], c.norm[dead], c.top[dead] = NAN, INF, NAN, NAN, NAN
    loss2, lse2 = c.loss()
    got = c.grad(lse3)
    torch.cuda.synchronize()
    assert torch.equal(loss, loss2) and torch.equal(lse, lse2)
    assert torch.equal(want[0], got[0]) and torch.equal(want[1], got[1])
    # words of -inf are no words
    c.ids[dead, 3], c.top[dead] = 5, -INF
    loss2, lse2 = c.loss()
    got = c.grad(lse3)
    torch.cuda.synchronize()
    assert torch.equal(loss, loss2) and torch.equal(lse, lse2)
    assert torch.equal(want[0], got[0]) and torch.equal(want[1], got[1])


def test_what_is_not_finite_stays_with_its_token(gpu):
    c = Case(gpu, 90, 700, 64, 9, absent=0.0, seed=8)
    loss, lse, first = c.loss(keep=True)
    dH, _ = c.grad(lse, head=False)
    c.top = c.top.clone()
    c.top[4, 2], c.top[60, 0] = NAN, INF
    loss2, lse2, kept = c.loss(keep=True)
    out = [c.grad(lse2, head=False, kept=k)[0] for k in (None, kept)]
    torch.cuda.synchronize()
    assert torch.equal(lse, lse2)
    odd = torch.zeros(90, dtype=torch.bool, device=gpu)
    odd[[4, 60]] = True
    assert loss2[odd].isnan().all() and torch.equal(loss2[~odd], loss[~odd])
    near, _ = c.grad(lse, head=False, kept=first)
    for x, want in zip(out, (dH, near)):
        assert x[odd].isnan().all() and torch.equal(x[~odd], want[~odd])


def test_words_that_the_student_rules_out(gpu):
    """z = -inf: probability 0. A teacher's word among them makes the loss infinite, of its token alone."""
    c = Case(gpu, 40, 1300, 64, 10, absent=0.0, seed=9)
    c.V[:, 0] = 0
    c.V[300:600, 0] = -INF
    c.H[:, 0] = 1
    c.ids = torch.where((c.ids >= 300) & (c.ids < 600), 7, c.ids)
    loss, lse, kept = c.loss(keep=True)
    out = [c.grad(lse, kept=k) for k in (None, kept)]
    torch.cuda.synchronize()
    keep = torch.cat([torch.arange(300), torch.arange(600, 1300)]).to(gpu)
    place = torch.full((1300,), -1, device=gpu)
    place[keep] = torch.arange(len(keep), device=gpu)
    small = Case(gpu, 40, 1300, 64, 10, absent=0.0, seed=9)
    small.H, small.V, small.ids = c.H, c.V[keep].contiguous(), place[c.ids.long()].int()
    _check_loss(small, loss, lse)
    for (dH, dV), k in zip(out, (False, True)):
        assert (dV[300:600] == 0).all()
        dH[:, 0] = 0  # (a sum of 0 times -inf)
        _check_grad(small, lse, dH, dV[keep], kept=k)
    c.ids[11, 3] = 450
    loss2, _ = c.loss()
    torch.cuda.synchronize()
    other = torch.arange(40, device=gpu) != 11
    assert float(loss2[11]) == INF and torch.equal(loss2[other], loss[other])


def test_a_word_past_the_vocabulary_is_reported(gpu):
    c = Case(gpu, 40, 300, 64, 6, seed=5)
    c.ids[7, 2], c.ids[9] = 300, 2 ** 31 - 1
    for call in (lambda err: c.loss(err=err), lambda err: c.grad(torch.zeros(40, device=gpu), err=err)):
        err = torch.zeros(1, dtype=torch.int32, device=gpu)
        call(err)
        torch.cuda.synchronize()
        assert int(err.item()) == bsq.DEVERR_BAD_SET
    loss, lse = c.loss()
    c.ids = torch.where(c.ids >= 300, -1, c.ids)
    c.live = (c.ids >= 0).any(1)
    _check_loss(c, loss, lse)
    err.zero_()
    c.loss(err=err)
    torch.cuda.synchronize()
    assert int(err.item()) == 0


def test_no_tokens(gpu):
    H, V = torch.empty((0, 64), dtype=torch.bfloat16, device=gpu), torch.randn((100, 64), device=gpu).bfloat16()
    ids, top = torch.empty((0, 5), dtype=torch.int32, device=gpu), torch.empty((0, 5), device=gpu)
    loss, lse, kept = bsq.bsq_distill_loss(H, V, ids, top, keep=True)
    assert loss.shape == (0,) and lse.shape == (0,)
    for k in (None, kept):
        dV = torch.ones_like(V)
        dH, _ = bsq.bsq_distill_grad(H, V, ids, top, lse, lse, kept=k, dV=dV)
        torch.cuda.synchronize()
        assert dH.shape == (0, 64) and (dV == 0).all()


def test_results_repeat_and_a_captured_step_replays(gpu):
    a = Case(gpu, 270, 2000, 200, 24, 0.2, seed=6)
    b = Case(gpu, 270, 2000, 200, 24, 0.5, seed=7)

    def step(c, stream=None):
        loss, lse, kept = c.loss(keep=True, stream=stream)
        return [loss, lse, *c.grad(lse, kept=kept, stream=stream), *c.grad(lse, stream=stream)]

    wants = [step(a), step(b)]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    other = step(a, side)
    side.synchronize()
    for q, w in zip(other, wants[0]):
        assert torch.equal(q, w)
    held_in = Case(gpu, 270, 2000, 200, 24, 0.2, seed=6)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = step(held_in)
    for c, want in ((a, wants[0]), (b, wants[1]), (a, wants[0])):
        for name in ("H", "V", "ids", "top", "g"):
            getattr(held_in, name).copy_(getattr(c, name))
        graph.replay()
        torch.cuda.synchronize()
        again = step(c)
        torch.cuda.synchronize()
        for q, w, x in zip(held, want, again):
            assert torch.equal(q, w) and torch.equal(x, w)


def test_kept_exponentials_past_32_bit_offsets(gpu):
    """8200 tokens of 270000 words: 2.2e9 exponentials, 4.4 GB. The last tokens by the definition."""
    T, N, D = 8200, 270000, 64
    c = Case(gpu, T, N, D, 16, seed=5)
    loss, lse, kept = c.loss(keep=True)
    dH, _ = c.grad(lse, kept=kept, head=False)
    last = slice(T - 20, T)
    c.H, c.ids, c.top, c.g = c.H[last], c.ids[last].contiguous(), c.top[last].contiguous(), c.g[last].contiguous()
    c.live = c.live[last]
    _check_loss(c, loss[last], lse[last])
    _check_grad(c, lse[last], dH[last], None, kept=True)
