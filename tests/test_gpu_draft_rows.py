"""Verification of drafted tokens where a block has several turns of a row and the row's
last turn is short: every word counts once. Against the definition in 64 bits, as in
test_gpu_draft.py; and with equal logits, where a probability is one over the number of
words."""
import pytest
import torch

import paper_2607_08643_amd as bsq
from parity_bounds import say
from test_gpu_draft import _case, _check, _reference

pytestmark = pytest.mark.gpu

INF = float("inf")

# B, L, N: rows that blocks have two or more turns of, whose last turn has 1 .. 2040 words,
# one word, all but one of a thread's, and whole vectors
SHAPES = [
    (64, 4, 50257),
    (64, 4, 49408),
    (64, 8, 131073),
    (256, 4, 33000),
    (300, 8, 24577),
    (1024, 2, 16385),
    (3000, 1, 8193),
    (64, 4, 151936),
    (600, 2, 12289),
]


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("B,L,N", SHAPES)
def test_every_word_counts_once(B, L, N, dt, gpu):
    """Equal logits: a certain draft is accepted below 1 / N; one drawn from the words of the
    second half alone below half / N. The random numbers lie 2^-10 below and above, where
    32-bit sums (2^-15) are sure."""
    say(f"draft rows B={B} L={L} N={N} {dt}")
    target = torch.zeros((1, 1, N), dtype=dt, device=gpu).expand(B, L + 1, N)
    half = torch.full((1, 1, N), -INF, dtype=dt, device=gpu)
    half[:, :, N // 2:] = 0.0
    tokens = torch.full((B, L), N - 1, dtype=torch.int32, device=gpu)
    want = torch.arange(B, device=gpu) % (L + 1)
    side = torch.where(torch.arange(L, device=gpu) < want[:, None], 1 - 2.0 ** -10, 1 + 2.0 ** -10)
    r = torch.zeros(B, device=gpu)
    for draft, share in ((None, 1 / N), (half.expand(B, L, N), (N - N // 2) / N)):
        count, out = bsq.bsq_draft_verify(target, tokens, (side * share).float(), r, draft)
        torch.cuda.synchronize()
        wrong = int((count != want).sum())
        say(f"  draft {draft is not None}: {wrong} of {B} sequences wrong")
        assert wrong == 0
        # the next token is the first of all, or of those that are left
        assert torch.equal(out.gather(1, want[:, None])[:, 0], torch.zeros_like(count))


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("B,L,N", [(64, 4, 50257), (256, 4, 33000), (100, 9, 24577)])
def test_many_long_rows_match_the_definition(B, L, N, dt, gpu):
    say(f"draft rows B={B} L={L} N={N} {dt}")
    target, tokens, u, r, draft, lens, temp = _case(gpu, B, L, N, dt, dt, seed=21)
    _check(_reference(target, tokens, u, r, draft), bsq.bsq_draft_verify(target, tokens, u, r, draft))
    temp[::3] = 0
    for given in (draft, None):
        _check(_reference(target, tokens, u, r, given, lens, temp),
               bsq.bsq_draft_verify(target, tokens, u, r, given, lens=lens, temperature=temp))


@pytest.mark.parametrize("rise", [1e-6, 1e-3, 20.0])
def test_rows_that_rise_over_many_turns(rise, gpu):
    """Rows whose every turn has a larger logit than those before, in blocks of 64 turns: random numbers next to
    the probability, further and further off."""
    say(f"draft rows that rise by {rise}")
    B, L, N = 512, 1, 1 << 20
    z = (torch.arange(N, dtype=torch.float64) / N * rise).float()
    target = z.to(gpu).expand(B, L + 1, N)
    token = torch.randint(0, N, (B, L), generator=torch.Generator().manual_seed(3))
    p = (z.double() - torch.logsumexp(z.double(), 0)).exp()
    off = torch.tensor([s * 2.0 ** -k for k in range(10, 23) for s in (1, -1)])
    u = (p[token[:, 0]] * (1 + off.repeat(B)[:B])).float()
    count, _ = bsq.bsq_draft_verify(target, token.int().to(gpu), u[:, None].to(gpu), torch.zeros(B, device=gpu))
    torch.cuda.synchronize()
    assert torch.equal(count.cpu() > 0, u.double() < p[token[:, 0]])
