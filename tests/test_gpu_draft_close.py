"""Draws from max(p - q, 0) where most words have p and q a few parts in 10^10 of each other:
which of them are above is decided by the rows' sums in 64 bits.

The target's and the draft's logits are equal but for one word of every 16, which holds
0.1 more in one row or the other, and for the last bits of one: the others have
p / q = 1 + (some 10^-10), and the first of them, word 0, is the first that a draw can
take. The sums of exponentials in 32 bits are some 10^-8 off, each row's in another
way. (The definition's own sums in 64 bits are off by 10^-15.)

The exponentials of 64 bits are off by 4e-14 of themselves, so are their sums, and p and q by 8e-14: a
cumulative sum of max(p - q, 0), of words that hold 1 of p and of q at most, by 1.6e-13, and
the number that it has to exceed by as much. The close words hold 4e-11 or more together."""
import pytest
import torch

import paper_2607_08643_amd as bsq
from parity_bounds import say
from test_gpu_draft import _law, _reference

pytestmark = pytest.mark.gpu

SLACK = 2 * 1.6e-13


def _rows(B, N, seed):
    """Target and draft logits [B, N] and a word with p < q."""
    g = torch.Generator().manual_seed(seed)
    word = torch.arange(N)
    group = (word // 8) % 2                       # alternate runs of eight
    z = torch.where(group == 0, 0.1, -0.7).repeat(B, 1) + 0.05 * torch.rand((B, 1), generator=g)
    special = (word % 4096 >= 2048) & (word % 8 == 3)
    a = 1 + torch.rand((B, 1), generator=g)
    b = a + 0.1
    p = torch.where(special, torch.where(group == 0, a, b), z)
    q = torch.where(special, torch.where(group == 0, b, a), z)
    at = int(special.nonzero()[-1])
    # the draft's sum a little larger
    q[:, at] += (torch.arange(B) % 4 + 1) * 2.0 ** -22
    return p, q, 2048 + 3


@pytest.mark.parametrize("N", [4096, 20480])
def test_words_next_to_the_border(N, gpu):
    B = 256
    p, q, token = _rows(B, N, 4)
    tokens = torch.full((B, 1), token, dtype=torch.int32)
    u = torch.full((B, 1), 1 - 2.0 ** -24)
    temp = 0.7 + torch.arange(B) / B * 0.6
    target, draft = torch.stack([p, p], 1), q[:, None].contiguous()
    # of the whole: nothing, some of the close words, the last of them, the others
    law = [(_law(p[b], temp[b]), _law(q[b], temp[b])) for b in range(B)]
    rest = torch.stack([(x - y).clamp_min(0) for x, y in law])
    close = rest.masked_fill(p != q, 0).sum(1) / rest.sum(1)
    say(f"  left of p: {float(rest.sum(1).min()):.4f} and more; close words hold {float(close.min()):.1e} to {float(close.max()):.1e} of it")
    assert (rest[:, 0] > 0).all() and rest.sum(1).min() > 2.0 ** -8
    for part in (0.0, 0.3, 0.9, 1.1, 1e6):
        r = (close * part).clamp(0, 0.9).float()
        want = _reference(target, tokens, u, r, draft, temperature=temp)
        assert (want[0] == 0).all()
        got = bsq.bsq_draft_verify(target.to(gpu), tokens.to(gpu), u.to(gpu), r.to(gpu), draft.to(gpu), temperature=temp.to(gpu))
        torch.cuda.synchronize()
        assert (got[0] == 0).all()
        word = got[1][:, :1].cpu().long()
        say(f"  at {part} of the close words' share: {int((word != want[1][:, :1]).sum())} of {B} draws are another word")
        if part == 0.0:
            assert (word == 0).all()
        sums = rest.cumsum(1)
        at = r.double() * sums[:, -1]
        upto = sums.gather(1, word)[:, 0]
        assert (rest.gather(1, word) > 0).all()
        assert (at < upto + SLACK).all() and (at >= upto - rest.gather(1, word)[:, 0] - SLACK).all()
