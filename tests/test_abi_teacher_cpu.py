"""The top-logit and draft-verification calls without a GPU: sizes, and every
refusal on the host before anything is launched (fake device pointers that are
never dereferenced)."""
import ctypes as ct

import pytest
import torch

import paper_2607_08643_amd as bsq

FAKE = 0x7F0000000000  # 256-aligned, never dereferenced: every call below fails validation first
BIG = 1 << 40


def _p(v):
    return ct.c_void_p(v) if v else None


# ---------------------------------------------------------------- top logits
def test_top_workspace():
    sizes = [bsq.bsq_top_workspace_bytes(T, N) for T, N in ((0, 1), (1, 1), (8, 151936), (512, 151936), (1 << 20, 151936))]
    assert all(0 < s <= 65 << 20 for s in sizes)
    for T, N, status in ((-1, 1, bsq.BSQ_ERR_SHAPE), (1, 0, bsq.BSQ_ERR_SHAPE), ((1 << 20) + 1, 1, bsq.BSQ_ERR_UNSUPPORTED),
                         (1, 1 << 31, bsq.BSQ_ERR_UNSUPPORTED)):
        with pytest.raises(bsq.BsqError) as e:
            bsq.bsq_top_workspace_bytes(T, N)
        assert e.value.status == status, (T, N)
    assert bsq.lib().bsq_top_workspace_bytes(1, 1, None) == bsq.BSQ_ERR_ARG


def test_top_rejects_before_launch():
    def call(Z=FAKE, dt=1, ldz=100, T=10, N=100, K=5, scale=1.0, ids=FAKE, top=FAKE, lse=FAKE, ws=FAKE, ws_bytes=BIG):
        return bsq.lib().bsq_top_logits(_p(Z), dt, ldz, T, N, K, scale, _p(ids), _p(top), _p(lse), _p(ws), ws_bytes, None)
    assert call(dt=2) == bsq.BSQ_ERR_DTYPE
    assert call(T=-1) == bsq.BSQ_ERR_SHAPE
    assert call(N=0) == bsq.BSQ_ERR_SHAPE
    assert call(ldz=99) == bsq.BSQ_ERR_SHAPE
    assert call(T=(1 << 20) + 1) == bsq.BSQ_ERR_UNSUPPORTED
    for K in (0, -1, 257):
        assert call(K=K) == bsq.BSQ_ERR_ARG
    for s in (0.0, -1.0, float("inf"), float("nan"), 2.0 ** -65, 2.0 ** 65):
        assert call(scale=s) == bsq.BSQ_ERR_ARG
    for kw in (dict(Z=0), dict(ids=0), dict(top=0), dict(ws=0)):
        assert call(**kw) == bsq.BSQ_ERR_ARG
    for kw in (dict(Z=FAKE + 1), dict(Z=FAKE + 2, dt=0), dict(ids=FAKE + 2), dict(top=FAKE + 1), dict(lse=FAKE + 2),
               dict(ws=FAKE + 128)):
        assert call(**kw) == bsq.BSQ_ERR_ALIGN, kw
    assert call(ws_bytes=bsq.bsq_top_workspace_bytes(10, 100) - 1) == bsq.BSQ_ERR_BUFFER_TOO_SMALL
    assert call(T=0, Z=0, ids=0, top=0, lse=0) == bsq.BSQ_OK  # nothing to do


# ---------------------------------------------------------------- drafts
def test_draft_workspace():
    assert bsq.bsq_draft_workspace_bytes(False, 64, 4, 151936) < bsq.bsq_draft_workspace_bytes(True, 64, 4, 151936) < 1 << 20
    bsq.bsq_draft_workspace_bytes(True, 0, 0, 1)
    for dims, status in (((-1, 1, 8), bsq.BSQ_ERR_SHAPE), ((1, -1, 8), bsq.BSQ_ERR_SHAPE), ((1, 1, 0), bsq.BSQ_ERR_SHAPE),
                         ((65537, 1, 8), bsq.BSQ_ERR_UNSUPPORTED), ((1, 65, 8), bsq.BSQ_ERR_UNSUPPORTED),
                         ((1, 1, 1 << 31), bsq.BSQ_ERR_UNSUPPORTED)):
        with pytest.raises(bsq.BsqError) as e:
            bsq.bsq_draft_workspace_bytes(True, *dims)
        assert e.value.status == status, dims
    out = ct.c_size_t(0)
    assert bsq.lib().bsq_draft_workspace_bytes(2, 1, 1, 1, ct.byref(out)) == bsq.BSQ_ERR_ARG
    assert bsq.lib().bsq_draft_workspace_bytes(1, 1, 1, 1, None) == bsq.BSQ_ERR_ARG


def test_draft_rejects_before_launch():
    def call(P=FAKE, pt=1, ps=300, pr=100, Q=FAKE, qt=1, qs=200, qr=100, B=3, L=2, N=100, tokens=FAKE, lens=0, u=FAKE,
             r=FAKE, temp=0, count=FAKE, out=FAKE, err=0, ws=FAKE, ws_bytes=BIG):
        return bsq.lib().bsq_draft_verify(_p(P), pt, ps, pr, _p(Q), qt, qs, qr, B, L, N, _p(tokens), _p(lens), _p(u), _p(r),
                                          _p(temp), _p(count), _p(out), _p(err), _p(ws), ws_bytes, None)
    assert call(pt=2) == bsq.BSQ_ERR_DTYPE
    assert call(qt=-1) == bsq.BSQ_ERR_DTYPE
    assert call(B=-1) == bsq.BSQ_ERR_SHAPE
    assert call(N=0) == bsq.BSQ_ERR_SHAPE
    assert call(L=65) == bsq.BSQ_ERR_UNSUPPORTED
    for kw in (dict(ps=-1), dict(pr=-1), dict(qs=-1), dict(qr=-1)):
        assert call(**kw) == bsq.BSQ_ERR_SHAPE, kw
    for kw in (dict(P=0), dict(tokens=0), dict(u=0), dict(r=0), dict(count=0), dict(out=0), dict(ws=0)):
        assert call(**kw) == bsq.BSQ_ERR_ARG, kw
    for kw in (dict(P=FAKE + 1), dict(P=FAKE + 2, pt=0), dict(Q=FAKE + 1), dict(Q=FAKE + 2, qt=0), dict(tokens=FAKE + 2),
               dict(lens=FAKE + 2), dict(u=FAKE + 2), dict(r=FAKE + 1), dict(temp=FAKE + 2), dict(count=FAKE + 2),
               dict(out=FAKE + 2), dict(err=FAKE + 1), dict(ws=FAKE + 64)):
        assert call(**kw) == bsq.BSQ_ERR_ALIGN, kw
    assert call(ws_bytes=bsq.bsq_draft_workspace_bytes(True, 3, 2, 100) - 1) == bsq.BSQ_ERR_BUFFER_TOO_SMALL
    # nothing of the draft is looked at where there is none; nothing to do without sequences
    assert call(Q=0, qt=9, qs=-1, qr=-1, ws_bytes=0) == bsq.BSQ_ERR_BUFFER_TOO_SMALL
    assert call(B=0, P=0, Q=0, tokens=0, u=0, r=0, count=0, out=0) == bsq.BSQ_OK


# ---------------------------------------------------------------- the binding's own checks
def test_binding_refuses_host_tensors_and_wrong_shapes():
    z = lambda *s, dt=torch.bfloat16: torch.zeros(s, dtype=dt)  # noqa: E731
    with pytest.raises(ValueError, match="GPU"):
        bsq.bsq_top_logits(z(4, 64), 3)
    with pytest.raises(TypeError, match="float16"):
        bsq.bsq_top_logits(z(4, 64, dt=torch.float16), 3)
    with pytest.raises(ValueError, match="contiguous"):
        bsq.bsq_top_logits(z(64, 4).T, 3)
    tokens, u, r = z(2, 3, dt=torch.int32), z(2, 3, dt=torch.float32), z(2, dt=torch.float32)
    with pytest.raises(ValueError, match="GPU"):
        bsq.bsq_draft_verify(z(2, 4, 50), tokens, u, r)
    with pytest.raises(ValueError, match="target"):
        bsq.bsq_draft_verify(z(2, 3, 50), tokens, u, r)
    with pytest.raises(ValueError, match="draft"):
        bsq.bsq_draft_verify(z(2, 4, 50), tokens, u, r, draft=z(2, 4, 50))
    with pytest.raises(ValueError, match="contiguous"):
        bsq.bsq_draft_verify(z(2, 50, 4).transpose(1, 2), tokens, u, r)
    with pytest.raises(TypeError, match="tokens"):
        bsq.bsq_draft_verify(z(2, 4, 50), tokens.long(), u, r)
    with pytest.raises(TypeError, match="u"):
        bsq.bsq_draft_verify(z(2, 4, 50), tokens, u.double(), r)
    with pytest.raises(ValueError, match="r"):
        bsq.bsq_draft_verify(z(2, 4, 50), tokens, u, u)
    with pytest.raises(ValueError, match="lens"):
        bsq.bsq_draft_verify(z(2, 4, 50), tokens, u, r, lens=z(3, dt=torch.int32))
    with pytest.raises(TypeError, match="temperature"):
        bsq.bsq_draft_verify(z(2, 4, 50), tokens, u, r, temperature=z(2))


# ---------------------------------------------------------------- distillation
@pytest.mark.parametrize("grad", [False, True])
def test_distill_workspace(grad):
    assert bsq.bsq_distill_workspace_bytes(grad, 0, 1, 8, 1) > 0
    assert bsq.bsq_distill_workspace_bytes(grad, 4096, 151936, 4096, 64) > bsq.bsq_xent_workspace_bytes(grad, 4096, 151936, 4096)
    for dims, status in (((-1, 1, 8, 1), bsq.BSQ_ERR_SHAPE), ((1, 0, 8, 1), bsq.BSQ_ERR_SHAPE), ((1, 1, 12, 1), bsq.BSQ_ERR_SHAPE),
                         ((1, 1, 8, 0), bsq.BSQ_ERR_ARG), ((1, 1, 8, 257), bsq.BSQ_ERR_ARG),
                         (((1 << 20) + 1, 1, 8, 1), bsq.BSQ_ERR_UNSUPPORTED), ((1, 1 << 31, 8, 1), bsq.BSQ_ERR_UNSUPPORTED)):
        with pytest.raises(bsq.BsqError) as e:
            bsq.bsq_distill_workspace_bytes(grad, *dims)
        assert e.value.status == status, dims
    assert 10 * 512 * 2 < bsq.bsq_distill_kept_bytes(10, 257, 64, 5) < bsq.bsq_distill_kept_bytes(300, 257, 64, 5)
    for dims in ((-1, 5, 8, 1), (1, 0, 8, 1), (1, 1, 8, 0)):
        with pytest.raises(bsq.BsqError):
            bsq.bsq_distill_kept_bytes(*dims)


def test_distill_rejects_before_launch():
    def call(grad, H=FAKE, ldh=64, V=FAKE, ldv=64, T=10, N=100, D=64, ids=FAKE, top=FAKE, norm=0, K=5, scale=1.0, a=FAKE,
             b=FAKE, kept=0, kept_bytes=0, dH=FAKE, lddh=64, dV=FAKE, lddv=64, dt=1, acc=0, err=0, ws=FAKE, ws_bytes=BIG):
        L = bsq.lib()
        if not grad:
            return L.bsq_distill_loss(_p(H), ldh, _p(V), ldv, T, N, D, _p(ids), _p(top), _p(norm), K, scale, _p(a), _p(b),
                                      _p(kept), kept_bytes, _p(err), _p(ws), ws_bytes, None)
        return L.bsq_distill_grad(_p(H), ldh, _p(V), ldv, T, N, D, _p(ids), _p(top), _p(norm), K, scale, _p(a), _p(b),
                                  _p(kept), kept_bytes, _p(dH), lddh, _p(dV), lddv, dt, acc, _p(err), _p(ws), ws_bytes, None)
    for g in (False, True):
        for kw in (dict(H=0), dict(V=0), dict(ids=0), dict(top=0), dict(a=0), dict(b=0), dict(ws=0), dict(K=0), dict(K=257),
                   dict(scale=0.0), dict(scale=-1.0), dict(scale=float("nan")), dict(scale=2.0 ** -65), dict(scale=2.0 ** 65)):
            assert call(g, **kw) == bsq.BSQ_ERR_ARG, kw
        for kw in (dict(T=-1), dict(N=0), dict(D=60), dict(ldh=63), dict(ldv=63), dict(ldv=68)):
            assert call(g, **kw) == bsq.BSQ_ERR_SHAPE, kw
        for kw in (dict(H=FAKE + 1), dict(V=FAKE + 8), dict(ids=FAKE + 2), dict(top=FAKE + 2), dict(norm=FAKE + 1),
                   dict(a=FAKE + 2), dict(b=FAKE + 2), dict(kept=FAKE + 16, kept_bytes=BIG), dict(err=FAKE + 2), dict(ws=FAKE + 64)):
            assert call(g, **kw) == bsq.BSQ_ERR_ALIGN, kw
        assert call(g, ws_bytes=bsq.bsq_distill_workspace_bytes(g, 10, 100, 64, 5) - 1) == bsq.BSQ_ERR_BUFFER_TOO_SMALL
        assert call(g, kept=FAKE, kept_bytes=bsq.bsq_distill_kept_bytes(10, 100, 64, 5) - 1) == bsq.BSQ_ERR_BUFFER_TOO_SMALL
    assert call(True, dH=0) == bsq.BSQ_ERR_ARG
    assert call(True, lddh=63) == bsq.BSQ_ERR_SHAPE
    assert call(True, lddv=63) == bsq.BSQ_ERR_SHAPE
    assert call(True, dt=5) == bsq.BSQ_ERR_DTYPE
    assert call(True, acc=-1) == bsq.BSQ_ERR_ARG
    assert call(True, dV=FAKE + 2, dt=0) == bsq.BSQ_ERR_ALIGN


def test_distill_binding_refuses_wrong_shapes():
    z = lambda *s, dt=torch.bfloat16: torch.zeros(s, dtype=dt)  # noqa: E731
    ids, top, f = z(4, 3, dt=torch.int32), z(4, 3, dt=torch.float32), z(4, dt=torch.float32)
    with pytest.raises(ValueError, match="GPU"):
        bsq.bsq_distill_loss(z(4, 64), z(10, 64), ids, top)
    with pytest.raises(TypeError, match="ids"):
        bsq.bsq_distill_loss(z(4, 64), z(10, 64), ids.long(), top)
    with pytest.raises(ValueError, match="K"):
        bsq.bsq_distill_loss(z(4, 64), z(10, 64), ids[0], top)
    with pytest.raises(ValueError, match="top"):
        bsq.bsq_distill_loss(z(4, 64), z(10, 64), ids, top[:, :2])
    with pytest.raises(ValueError, match="norm"):
        bsq.bsq_distill_loss(z(4, 64), z(10, 64), ids, top, norm=top)
    with pytest.raises(ValueError, match="accumulate"):
        bsq.bsq_distill_grad(z(4, 64), z(10, 64), ids, top, f, f, accumulate=True)
    with pytest.raises(TypeError, match="g"):
        bsq.bsq_distill_grad(z(4, 64), z(10, 64), ids, top, f, f.double())
