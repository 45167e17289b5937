"""Rows of H, dH and dV at any alignment of their elements: the same bits as
aligned rows, and nothing between the rows is touched."""
import pytest
import torch

import paper_2607_08643_amd as bsq
from parity_bounds import say
from test_gpu_xent import _inputs, _weights

pytestmark = pytest.mark.gpu

FILL = 7.0


def _rows(rows, cols, pad, offset, dtype, gpu):
    """A view of rows `pad` elements apart beyond their width, from an element
    offset on, and the buffer around it."""
    buf = torch.full((rows * (cols + pad) + offset,), FILL, dtype=dtype, device=gpu)
    return buf[offset:].view(rows, cols + pad)[:, :cols], buf


def _gaps_untouched(view, buf):
    again = torch.full_like(buf, FILL)
    at = (view.data_ptr() - buf.data_ptr()) // buf.element_size()
    again[at:].view(view.shape[0], view.stride(0))[:, :view.shape[1]] = view
    return torch.equal(again, buf)


@pytest.mark.parametrize("pad,offset", [(1, 0), (3, 1), (0, 1), (2, 2), (4, 4)])
@pytest.mark.parametrize("T,N,D,ignore", [(7, 300, 72, 0.0), (70, 513, 200, 0.3), (1100, 700, 64, 0.1)])
def test_rows_at_odd_places(T, N, D, ignore, pad, offset, gpu):
    say(f"xent rows T={T} N={N} D={D} pad={pad} offset={offset}")
    H, V, target = _inputs(gpu, T, N, D, ignore, seed=14)
    g = _weights(T, 5, gpu)
    X, _ = _rows(T, D, pad, offset, torch.bfloat16, gpu)
    X.copy_(H)
    loss, lse = bsq.bsq_xent_loss(H, V, target)
    loss2, lse2 = bsq.bsq_xent_loss(X, V, target)
    torch.cuda.synchronize()
    assert torch.equal(loss, loss2) and torch.equal(lse, lse2)
    for dt in (torch.bfloat16, torch.float32):
        for accumulate in (False, True):
            start = torch.randn((N, D), generator=torch.Generator().manual_seed(3)).to(dt).to(gpu)
            want = start.clone()
            dH, _ = bsq.bsq_xent_grad(H, V, target, lse, g, dV=want, accumulate=accumulate)
            dX, around_x = _rows(T, D, pad, offset, torch.bfloat16, gpu)
            dW, around_w = _rows(N, D, pad, offset, dt, gpu)
            dW.copy_(start)
            bsq.bsq_xent_grad(X, V, target, lse, g, dH=dX, dV=dW, accumulate=accumulate)
            torch.cuda.synchronize()
            assert torch.equal(dX, dH) and torch.equal(dW, want)
            assert _gaps_untouched(dX, around_x) and _gaps_untouched(dW, around_w)
