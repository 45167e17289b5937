"""Draws from vocabularies past 2^21 words (a wave's part of a row is then longer than one
of its turns), and draws where nothing is left of max(p - q, 0)."""
import pytest
import torch

import paper_2607_08643_amd as bsq
from parity_bounds import say
from test_gpu_draft import _case, _check, _law, _reference

pytestmark = pytest.mark.gpu

INF = float("inf")


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("B,L,N", [(3, 1, (1 << 21) + 1), (2, 1, 2200003), (1, 1, (1 << 22) + 777), (2, 0, 5000011)])
def test_runs_of_several_turns(B, L, N, dt, gpu):
    say(f"draft B={B} L={L} N={N} {dt}")
    for seed in (1, 2):
        target, tokens, u, r, draft, lens, temp = _case(gpu, B, L, N, dt, dt, seed=seed)
        if L:
            u[0] = 1 - 2.0 ** -24
        _check(_reference(target, tokens, u, r, draft), bsq.bsq_draft_verify(target, tokens, u, r, draft))
        _check(_reference(target, tokens, u, r, None, None, temp), bsq.bsq_draft_verify(target, tokens, u, r, temperature=temp))
    # the last word and the first
    r[:] = 1 - 2.0 ** -24
    r[0] = 0.0
    _check(_reference(target, tokens, u, r, draft), bsq.bsq_draft_verify(target, tokens, u, r, draft))


@pytest.mark.parametrize("pt,qt", [(torch.bfloat16, torch.bfloat16), (torch.float32, torch.float32), (torch.float32, torch.bfloat16)])
@pytest.mark.parametrize("N", [3, 700, 9001])
def test_nothing_left_draws_from_the_target(N, pt, qt, gpu):
    """The draft's logits are the target's, and the drafted token is masked in both: it is refused with
    any random number, and nothing is left of max(p - q, 0)."""
    say(f"draft N={N} {pt} {qt}")
    g = torch.Generator().manual_seed(3)
    B = 40
    z = (torch.randn((B, 2, N), generator=g) * 2).bfloat16()
    tokens = torch.randint(0, N, (B, 1), generator=g)
    z[torch.arange(B), 0, tokens[:, 0]] = -INF
    target, draft = z.to(pt).to(gpu), z[:, :1].to(qt).to(gpu)
    u, r = torch.zeros((B, 1), device=gpu), torch.rand(B, generator=g).to(gpu)
    err = torch.zeros(1, dtype=torch.int32, device=gpu)
    count, out = bsq.bsq_draft_verify(target, tokens.int().to(gpu), u, r, draft, err=err)
    torch.cuda.synchronize()
    want = []
    for b in range(B):
        sums = _law(z[b, 0], 1.0).cumsum(0)
        want.append(int((sums <= float(r[b]) * float(sums[-1])).sum()))
    assert count.tolist() == [0] * B and out.tolist() == [[w, -1] for w in want] and int(err.item()) == 0
