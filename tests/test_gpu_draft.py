"""Verification of drafted tokens (bsq_draft_verify) against the definition in 64
bits, one sequence and one token after another. Results are whole numbers and have to
be equal: both are those of 64-bit sums, so a draw on a vocabulary of N words differs
only where a random number lies within some 1e-13 of a border of the cumulative sum."""
import pytest
import torch

import paper_2607_08643_amd as bsq
from parity_bounds import say

pytestmark = pytest.mark.gpu

INF, NAN = float("inf"), float("nan")


def _law(z, tau):
    x = z.double() / tau
    e = (x - x.max()).exp()
    return e / e.sum()


def _largest(z):
    z = z.float()
    return int((z == z.max()).nonzero()[0])


def _reference(target, tokens, u, r, draft=None, lens=None, temperature=None):
    target, tokens = target.cpu(), tokens.cpu()
    draft = None if draft is None else draft.cpu()
    B, L = tokens.shape
    count, out = [], []
    for b in range(B):
        n = L if lens is None else int(lens[b])
        tau = 1.0 if temperature is None else float(temperature[b])
        said, w = [], None
        for i, x in enumerate(tokens[b, :n].tolist()):
            if tau == 0:
                if _largest(target[b, i]) != x:
                    break
            else:
                p = _law(target[b, i], tau)
                if draft is None:
                    q = torch.zeros_like(p)
                    q[x] = 1.0
                else:
                    q = _law(draft[b, i], tau)
                if not float(u[b, i]) * float(q[x]) < float(p[x]):
                    w = (p - q).clamp_min(0)
                    if float(w.sum()) == 0:
                        w = p
                    break
            said.append(x)
        if tau == 0:
            nxt = _largest(target[b, len(said)])
        else:
            sums = (_law(target[b, len(said)], tau) if w is None else w).cumsum(0)
            nxt = int((sums <= float(r[b]) * float(sums[-1])).sum())
        count.append(len(said))
        out.append(said + [nxt] + [-1] * (L - len(said)))
    return torch.tensor(count, dtype=torch.int32), torch.tensor(out, dtype=torch.int32).view(B, L + 1)


def _case(gpu, B, L, N, pt=torch.bfloat16, qt=torch.bfloat16, near=0.7, masked=0.0, seed=1):
    g = torch.Generator().manual_seed(seed)
    z = torch.randn((B, L + 1, N), generator=g) * 2.5
    if masked:
        z[torch.rand(z.shape, generator=g) < masked] = -INF
        z[:, :, N // 2] = 0.0
    y = z[:, :L] + near * torch.randn((B, L, N), generator=g)
    target, draft = z.to(pt), y.to(qt)
    noise = -(-torch.rand((B, L, N), generator=g).clamp(1e-7, 1 - 1e-7).log()).log()
    tokens = (draft.float() + noise).argmax(2).int() if L else torch.empty((B, 0), dtype=torch.int32)
    u, r = torch.rand((B, L), generator=g), torch.rand(B, generator=g)
    lens = torch.randint(0, L + 1, (B,), generator=g).int()
    temp = torch.rand(B, generator=g) + 0.5
    return [t.to(gpu) for t in (target, tokens, u, r, draft, lens, temp)]


def _check(want, got):
    torch.cuda.synchronize()
    assert torch.equal(got[0].cpu(), want[0])
    assert torch.equal(got[1].cpu(), want[1])


SHAPES = [
    # B, L, N
    (1, 0, 1),
    (1, 1, 1),
    (3, 0, 1000),
    (2, 1, 7),
    (5, 3, 129),
    (17, 4, 2049),
    (4, 8, 8191),
    (2, 64, 300),
    (3, 2, 8193),
    (6, 5, 32003),
    (2, 4, 151936),
    (1, 1, 600001),
]


@pytest.mark.parametrize("pt,qt", [(torch.bfloat16, torch.bfloat16), (torch.float32, torch.float32),
                                   (torch.bfloat16, torch.float32), (torch.float32, torch.bfloat16)])
@pytest.mark.parametrize("B,L,N", SHAPES)
def test_matches_definition(B, L, N, pt, qt, gpu):
    say(f"draft B={B} L={L} N={N} {pt} {qt}")
    target, tokens, u, r, draft, lens, temp = _case(gpu, B, L, N, pt, qt)
    _check(_reference(target, tokens, u, r, draft), bsq.bsq_draft_verify(target, tokens, u, r, draft))
    _check(_reference(target, tokens, u, r, None, lens, temp),
           bsq.bsq_draft_verify(target, tokens, u, r, lens=lens, temperature=temp))
    temp[::2] = 0
    _check(_reference(target, tokens, u, r, draft, lens, temp),
           bsq.bsq_draft_verify(target, tokens, u, r, draft, lens=lens, temperature=temp))


@pytest.mark.parametrize("near", [0.0, 0.05, 3.0])
@pytest.mark.parametrize("masked", [0.0, 0.95])
def test_near_and_far_drafts(near, masked, gpu):
    """Drafts that are the target's own, nearly so, and far from it; most words masked."""
    for seed in range(3):
        target, tokens, u, r, draft, lens, temp = _case(gpu, 20, 5, 3001, near=near, masked=masked, seed=seed)
        want = _reference(target, tokens, u, r, draft, lens, temp)
        _check(want, bsq.bsq_draft_verify(target, tokens, u, r, draft, lens=lens, temperature=temp))
        if near == 0.0:
            assert torch.equal(want[0], lens.cpu())
        say(f"  near={near} masked={masked}: accepted {float(want[0].float().mean()):.2f} of {float(lens.float().mean()):.2f}")


def test_random_numbers_on_borders(gpu):
    """Probabilities that are powers of two: the comparison is strict, a cumulative sum has to exceed."""
    last = 1 - 2.0 ** -24
    target = torch.zeros((6, 2, 8), device=gpu)
    draft = torch.full((6, 1, 8), -INF, device=gpu)
    draft[:, 0, :4] = 1.0                     # 1/4 on four words; the target 1/8 on eight
    tokens = torch.full((6, 1), 2, dtype=torch.int32, device=gpu)
    u = torch.tensor([0.5, 0.5 - 2.0 ** -25, 0.0, last, last, 0.75], device=gpu)[:, None]
    r = torch.tensor([0.0, 0.25, last, 0.5, last, 0.25 - 2.0 ** -26], device=gpu)
    count, out = bsq.bsq_draft_verify(target, tokens, u, r, draft)
    torch.cuda.synchronize()
    assert count.tolist() == [0, 1, 1, 0, 0, 0]
    # refused: from 1/8 on words 4 .. 7; accepted: from 1/8 on all
    assert out.tolist() == [[4, -1], [2, 2], [2, 7], [6, -1], [7, -1], [4, -1]]
    # a draft that is the target: accepted with any u
    count, out = bsq.bsq_draft_verify(target, tokens, torch.full_like(u, last), r, target[:, :1].clone())
    torch.cuda.synchronize()
    assert (count == 1).all()


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32])
def test_random_numbers_next_to_the_ratio(dt, gpu):
    """u is p / q rounded to 32 bits, and its neighbours: 32-bit sums do not settle any of these."""
    target, tokens, u, r, draft, lens, temp = _case(gpu, 12, 4, 5003, dt, dt, near=0.4, seed=13)
    for given in (draft, None):
        for b in range(12):
            for i in range(4):
                x, tau = int(tokens[b, i]), float(temp[b])
                p = _law(target[b, i].cpu(), tau)[x]
                q = _law(draft[b, i].cpu(), tau)[x] if given is not None else torch.tensor(1.0)
                u[b, i] = min(float(p / q), 1 - 2.0 ** -24)
        for side in (0.0, 1.0, -1.0):
            v = torch.nextafter(u, torch.full_like(u, side * 2)) if side else u
            v = v.clamp(0, 1 - 2.0 ** -24)
            _check(_reference(target, tokens, v, r, given, lens, temp),
                   bsq.bsq_draft_verify(target, tokens, v, r, given, lens=lens, temperature=temp))


@pytest.mark.parametrize("near", [1e-5, 1e-3, 2e-2])
def test_little_left_of_the_target(near, gpu):
    """Drafts so near to the target that max(p - q, 0) is a small part of p, and refused all the same."""
    target, tokens, u, r, draft, lens, temp = _case(gpu, 40, 2, 4001, torch.float32, torch.float32, near=near, seed=14)
    parts = []
    for b in range(40):
        for i in range(2):
            x, tau = int(tokens[b, i]), float(temp[b])
            p, q = _law(target[b, i].cpu(), tau), _law(draft[b, i].cpu(), tau)
            u[b, i] = 1 - 2.0 ** -24 if p[x] < q[x] else 0.0
            parts.append(float((p - q).clamp_min(0).sum()))
    want = _reference(target, tokens, u, r, draft, lens, temp)
    say(f"  near={near}: max(p - q, 0) is {min(parts):.1e} to {max(parts):.1e}; accepted {int(want[0].sum())} of {int(lens.sum())}")
    assert (want[0] < lens.cpu()).any()
    _check(want, bsq.bsq_draft_verify(target, tokens, u, r, draft, lens=lens, temperature=temp))


@pytest.mark.parametrize("tau", [1e-30, 1e-6, 0.01, 50.0, 1e10])
def test_temperatures_of_any_size(tau, gpu):
    target, tokens, u, r, draft, lens, _ = _case(gpu, 16, 3, 3000, masked=0.3, seed=15)
    temp = torch.full((16,), tau, device=gpu)
    want_temp = temp if tau > 2.0 ** -64 else torch.zeros_like(temp)  # (smaller ones count as 0)
    _check(_reference(target, tokens, u, r, draft, lens, want_temp),
           bsq.bsq_draft_verify(target, tokens, u, r, draft, lens=lens, temperature=temp))


def test_outputs_follow_the_target(gpu):
    """Whatever the draft, the first token out is distributed as the target's: 40000 sequences, each word's share
    within five standard deviations."""
    B, N = 40000, 12
    g = torch.Generator().manual_seed(3)
    z, y = torch.randn((1, 2, N), generator=g), torch.randn((1, 1, N), generator=g)
    q = _law(y[0, 0], 1.0)
    tokens = torch.multinomial(q, B, replacement=True, generator=g).int()[:, None].to(gpu)
    u, r = torch.rand((B, 1), generator=g).to(gpu), torch.rand(B, generator=g).to(gpu)
    for draft in (True, False):
        if not draft:
            tokens = torch.full_like(tokens, 3)
        count, out = bsq.bsq_draft_verify(z.to(gpu).expand(B, 2, N), tokens, u, r,
                                          draft=y.to(gpu).expand(B, 1, N) if draft else None)
        torch.cuda.synchronize()
        share = torch.bincount(out[:, 0].long().cpu(), minlength=N).double() / B
        p = _law(z[0, 0], 1.0)
        off = (share - p).abs() / (p * (1 - p) / B).sqrt()
        say(f"  worst {float(off.max()):.2f} standard deviations; accepted {float(count.float().mean()):.3f}")
        assert (off < 5).all()


def test_equal_logits_take_the_lowest_word(gpu):
    target = torch.zeros((2, 3, 9000), dtype=torch.bfloat16, device=gpu)
    target[:, 0, [40, 41, 8999]] = 7.0
    tokens = torch.tensor([[40, 0], [41, 0]], dtype=torch.int32, device=gpu)
    u, r = torch.zeros((2, 2), device=gpu), torch.zeros(2, device=gpu)
    count, out = bsq.bsq_draft_verify(target, tokens, u, r, temperature=torch.zeros(2, device=gpu))
    torch.cuda.synchronize()
    assert count.tolist() == [2, 0] and out.tolist() == [[40, 0, 0], [40, -1, -1]]


def test_rows_without_a_probability(gpu):
    target, tokens, u, r, draft, _, _ = _case(gpu, 7, 3, 2500, near=0.0, seed=6)
    want = _reference(target, tokens, u, r, draft)
    target[1, 1, 77] = NAN
    target[2, 3, 5] = INF
    target[3, 0] = -INF
    draft[4, 2, 9] = NAN
    lens = torch.tensor([3, 3, 3, 3, 3, 1, 0], dtype=torch.int32, device=gpu)
    target[5, 2], draft[5, 1], target[6, 1:], draft[6] = NAN, NAN, NAN, NAN  # past the drafted tokens
    for temp in (None, torch.zeros(7, device=gpu)):
        err = torch.zeros(1, dtype=torch.int32, device=gpu)
        count, out = bsq.bsq_draft_verify(target, tokens, u, r, draft, lens=lens, temperature=temp, err=err)
        torch.cuda.synchronize()
        assert int(err.item()) == bsq.DEVERR_NONFINITE
        if temp is not None:
            # (greedy: +inf is the largest; nothing is drafted from NaN)
            assert out[3].tolist() == [-1] * 4 and int(count[3]) == 0
            continue
        assert count.tolist() == [3, 1, 3, 0, 2, 1, 0]
        assert out[0].tolist() == want[1][0].tolist()
        assert out[1].tolist() == [int(tokens[1, 0]), -1, -1, -1]
        assert out[2].tolist() == tokens[2].tolist() + [-1]
        assert out[3].tolist() == [-1] * 4
        drawn = _law(target[4, 2].cpu(), 1.0).cumsum(0)
        assert int(out[4, 2]) == int((drawn <= float(r[4]) * float(drawn[-1])).sum())
        assert out[5, 0] == tokens[5, 0] and 0 <= int(out[5, 1]) < 2500 and out[5, 2:].tolist() == [-1, -1]
        assert 0 <= int(out[6, 0]) < 2500
    err.zero_()
    bsq.bsq_draft_verify(target[:1], tokens[:1], u[:1], r[:1], draft[:1], err=err)
    torch.cuda.synchronize()
    assert int(err.item()) == 0


def test_tokens_lengths_and_temperatures_out_of_range(gpu):
    target, tokens, u, r, draft, _, _ = _case(gpu, 6, 3, 700, near=0.0, seed=2)
    u.zero_()
    base = tokens.clone()
    lens = torch.tensor([3, 3, 9, -2, 3, 3], dtype=torch.int32, device=gpu)
    temp = torch.tensor([1.0, 1.0, 1.0, 1.0, -1.0, NAN], device=gpu)
    tokens[0, 1], tokens[1, 0] = 700, -1
    for given in (draft, None):
        err = torch.zeros(1, dtype=torch.int32, device=gpu)
        count, out = bsq.bsq_draft_verify(target, tokens, u, r, given, lens=lens, temperature=temp, err=err)
        torch.cuda.synchronize()
        assert int(err.item()) == bsq.DEVERR_BAD_SET
        assert count[:4].tolist() == [1, 0, 3, 0]
        greedy = bsq.bsq_draft_verify(target, base, u, r, given, temperature=torch.zeros(6, device=gpu))
        torch.cuda.synchronize()
        assert torch.equal(out[4:], greedy[1][4:]) and torch.equal(count[4:], greedy[0][4:])
        # a token outside the vocabulary takes no word out of the draw
        if given is None:
            sums = _law(target[1, 0].cpu(), 1.0).cumsum(0)
            assert int(out[1, 0]) == int((sums <= float(r[1]) * float(sums[-1])).sum())


def test_strides_and_offsets_past_32_bits(gpu):
    B, L, N = 2, 2, 900
    target, tokens, u, r, draft, lens, temp = _case(gpu, B, L, N, seed=11)
    want = _reference(target, tokens, u, r, draft)
    row = (1 << 30) + 3
    big = torch.empty(5 * row + N + 1, dtype=torch.bfloat16, device=gpu)
    P = big[1:].as_strided((B, L + 1, N), (3 * row, row, 1))
    P.copy_(target)
    buf = torch.full((L, B, N + 7), NAN, dtype=torch.bfloat16, device=gpu)
    Q = buf[:, :, 3:3 + N].transpose(0, 1)
    Q.copy_(draft)
    _check(want, bsq.bsq_draft_verify(P, tokens, u, r, Q))


def test_no_sequences(gpu):
    z = torch.empty((0, 4, 100), device=gpu)
    count, out = bsq.bsq_draft_verify(z, torch.empty((0, 3), dtype=torch.int32, device=gpu), torch.empty((0, 3), device=gpu),
                                      torch.empty(0, device=gpu))
    assert count.shape == (0,) and out.shape == (0, 4)


def test_another_stream_and_a_captured_call(gpu):
    a = _case(gpu, 9, 4, 20011, seed=1)
    b = _case(gpu, 9, 4, 20011, seed=2)

    def call(c, stream=None):
        target, tokens, u, r, draft, lens, temp = c
        return bsq.bsq_draft_verify(target, tokens, u, r, draft, lens=lens, temperature=temp, stream=stream)

    wa, wb = call(a), call(b)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = call(a, side)
    side.synchronize()
    assert torch.equal(got[0], wa[0]) and torch.equal(got[1], wa[1])
    held_in = [t.clone() for t in a]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = call(held_in)
    for src, want in ((a, wa), (b, wb), (a, wa)):
        for h, s in zip(held_in, src):
            h.copy_(s)
        graph.replay()
        torch.cuda.synchronize()
        again = call(src)
        torch.cuda.synchronize()
        for h, w, x in zip(held, want, again):
            assert torch.equal(h, w) and torch.equal(x, w)


def test_the_largest_batch(gpu):
    say("draft B=65536 L=1 N=2")
    g = torch.Generator().manual_seed(3)
    B = 65536
    target, u, r = torch.randn((B, 2, 2), generator=g), torch.rand((B, 1), generator=g), torch.rand(B, generator=g)
    tokens = torch.randint(0, 2, (B, 1), generator=g).int()
    p = target.double().softmax(2)
    kept = u[:, 0].double() < p[:, 0].gather(1, tokens.long())[:, 0]
    # refused: the other word is all that is left
    after = torch.where(p[:, 1, 0] > r.double(), 0, 1)
    want = torch.stack([torch.where(kept, tokens[:, 0], 1 - tokens[:, 0]), torch.where(kept, after, -1)], 1).int()
    _check((kept.int(), want), bsq.bsq_draft_verify(target.to(gpu), tokens.to(gpu), u.to(gpu), r.to(gpu)))


def test_rows_that_sequences_share(gpu):
    say("draft rows of stride 0")
    target, tokens, u, r, draft, lens, temp = _case(gpu, 6, 3, 1001)
    one, two = target[:1].expand(6, 4, 1001), draft[:, :1].expand(6, 3, 1001)
    _check(_reference(one, tokens, u, r, two, lens, temp),
           bsq.bsq_draft_verify(one, tokens, u, r, two, lens=lens, temperature=temp))


def test_two_streams_at_once(gpu):
    say("draft and top logits on two streams")
    target, tokens, u, r, draft, lens, temp = _case(gpu, 5, 4, 32003)
    want = _reference(target, tokens, u, r, draft)
    ids, top, lse = bsq.bsq_top_logits(target[:, 0], 40)
    one, two = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    got = []
    for _ in range(4):
        with torch.cuda.stream(one):
            verified = bsq.bsq_draft_verify(target, tokens, u, r, draft)
        with torch.cuda.stream(two):
            listed = bsq.bsq_top_logits(target[:, 0], 40)
        got.append((verified, listed))
    torch.cuda.synchronize()
    for verified, listed in got:
        _check(want, verified)
        assert all(torch.equal(x, y) for x, y in zip(listed, (ids, top, lse)))
