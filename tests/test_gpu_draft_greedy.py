"""Verification of drafted tokens at temperature 0 where target rows hold what is not finite:
+inf is the largest (of several the lowest word), a NaN leaves the row without a word.
One sequence a call, so that every case has the error word to itself."""
import pytest
import torch

import paper_2607_08643_amd as bsq

pytestmark = pytest.mark.gpu

INF, NAN = float("inf"), float("nan")


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("N", [5, 2500, 40000])
def test_greedy_rows_that_are_not_finite(N, dt, gpu):
    g = torch.Generator().manual_seed(2)
    base = torch.randn((1, 4, N), generator=g).to(dt)
    best = base.float()[0].argmax(1).tolist()
    u, r, temp = torch.zeros((1, 3), device=gpu), torch.zeros(1, device=gpu), torch.zeros(1, device=gpu)

    def call(z, tokens):
        err = torch.zeros(1, dtype=torch.int32, device=gpu)
        draft = torch.full((1, 3, N), NAN, dtype=dt, device=gpu)  # not used
        got = [bsq.bsq_draft_verify(z.to(gpu), torch.tensor([tokens], dtype=torch.int32, device=gpu), u, r, draft=d,
                                    temperature=temp, err=err) for d in (None, draft)]
        torch.cuda.synchronize()
        assert got[0][0].tolist() == got[1][0].tolist() and got[0][1].tolist() == got[1][1].tolist()
        return got[0][0].tolist()[0], got[0][1].tolist()[0], int(err.item())

    assert call(base, best[:3]) == (3, best, 0)
    for row in range(4):
        for place in (0, N // 2, N - 1):
            said = best[:row]
            z = base.clone()
            z[0, row, place] = NAN
            assert call(z, best[:3]) == (row, said + [-1] * (4 - row), bsq.DEVERR_NONFINITE)
            z[0, row] = -INF
            assert call(z, best[:3]) == (row, said + [-1] * (4 - row), bsq.DEVERR_NONFINITE)
            # +inf: accepted, where it was drafted, else what follows
            z = base.clone()
            z[0, row, place], z[0, row, N - 1] = INF, INF
            with_it = best[:row] + [place] + best[row + 1:]
            assert call(z, with_it[:3]) == (3, with_it, 0)
            if row < 3:
                other = best[:row] + [(place + 1) % N] + best[row + 1:]
                assert call(z, other[:3]) == (row, said + [place] + [-1] * (3 - row), 0)
            # past the first refusal nothing counts
            if row:
                z[0, row, place] = NAN
                wrong = [(best[0] + 1) % N] + best[1:]
                assert call(z, wrong[:3]) == (0, [best[0], -1, -1, -1], 0)
