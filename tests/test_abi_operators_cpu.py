"""The adapter, cross-entropy and clipping calls without a GPU: sizes, and every
refusal on the host before anything is launched (fake device pointers that are
never dereferenced)."""
import ctypes as ct

import pytest
import torch

import paper_2607_08643_amd as bsq
from paper_2607_08643_amd import _binding as B

FAKE = 0x7F0000000000  # 256-aligned, never dereferenced: every call below fails validation first
BIG = 1 << 40
P = ct.c_void_p


def _p(v):
    return P(v) if v else None


def _arr(*v):
    return (P * len(v))(*[x or None for x in v])


def _i64(*v):
    return (ct.c_int64 * len(v))(*v)


# ---------------------------------------------------------------- adapters
def _plan(M=1000, n=4, ids=FAKE, buf=FAKE):
    return B.bsq_adapter_plan(ids or None, buf or None, M, n)


def _pool(A=FAKE, Bp=FAKE, scale=0, ranks=0, d_out=64):
    return (B.bsq_adapter_pool * 1)(B.bsq_adapter_pool(A or None, Bp or None, scale or None, ranks or None, d_out))


def test_adapter_plan_sizes_and_refusals():
    Lib = bsq.lib()
    sizes = [bsq.bsq_adapters_plan_bytes(M, n) for M, n in ((1, 1), (256, 1024), (257, 1), (1000, 16), (1000, 1024), (1 << 24, 1024))]
    assert sizes == sorted(sizes) and sizes[1] == 0 and sizes[2] > 0  # up to 256 tokens there is nothing to keep
    for M, n, status in ((0, 1, bsq.BSQ_ERR_SHAPE), (-1, 1, bsq.BSQ_ERR_SHAPE), (1, 0, bsq.BSQ_ERR_SHAPE),
                         ((1 << 24) + 1, 1, bsq.BSQ_ERR_UNSUPPORTED), (1, 1025, bsq.BSQ_ERR_UNSUPPORTED)):
        with pytest.raises(bsq.BsqError) as e:
            bsq.bsq_adapters_plan_bytes(M, n)
        assert e.value.status == status

    def plan(p, nbytes=BIG, err=0):
        return Lib.bsq_adapters_plan(ct.byref(p), nbytes, _p(err), None)
    assert Lib.bsq_adapters_plan(None, BIG, None, None) == bsq.BSQ_ERR_ARG
    assert plan(_plan(ids=0)) == bsq.BSQ_ERR_ARG
    assert plan(_plan(buf=0)) == bsq.BSQ_ERR_ARG
    assert plan(_plan(M=0)) == bsq.BSQ_ERR_SHAPE
    assert plan(_plan(n=2000)) == bsq.BSQ_ERR_UNSUPPORTED
    assert plan(_plan(ids=FAKE + 2)) == bsq.BSQ_ERR_ALIGN
    assert plan(_plan(buf=FAKE + 8)) == bsq.BSQ_ERR_ALIGN
    assert plan(_plan(), err=FAKE + 1) == bsq.BSQ_ERR_ALIGN
    assert plan(_plan(), nbytes=bsq.bsq_adapters_plan_bytes(1000, 4) - 1) == bsq.BSQ_ERR_BUFFER_TOO_SMALL
    assert Lib.bsq_adapters_plan_bytes(1, 1, None) == bsq.BSQ_ERR_ARG


@pytest.mark.parametrize("back", [False, True])
def test_adapter_workspace(back):
    one = bsq.bsq_adapters_workspace_bytes(back, 100, 4, 16, 256, [64])
    assert 0 < one < bsq.bsq_adapters_workspace_bytes(back, 4000, 4, 128, 4096, [4096, 1024])
    for kw, status in ((dict(M=0), bsq.BSQ_ERR_SHAPE), (dict(n=0), bsq.BSQ_ERR_SHAPE), (dict(rank=0), bsq.BSQ_ERR_ARG),
                       (dict(rank=129), bsq.BSQ_ERR_ARG), (dict(d_in=0), bsq.BSQ_ERR_SHAPE),
                       (dict(d_out=[0]), bsq.BSQ_ERR_SHAPE), (dict(d_out=[64] * 9), bsq.BSQ_ERR_ARG),
                       (dict(d_out=[]), bsq.BSQ_ERR_ARG), (dict(d_in=(1 << 24) + 1), bsq.BSQ_ERR_UNSUPPORTED),
                       (dict(d_out=[1 << 25]), bsq.BSQ_ERR_UNSUPPORTED)):
        a = dict(M=100, n=4, rank=16, d_in=256, d_out=[64])
        a.update(kw)
        with pytest.raises(bsq.BsqError) as e:
            bsq.bsq_adapters_workspace_bytes(back, **a)
        assert e.value.status == status, kw


def test_adapters_apply_rejects_before_launch():
    Lib = bsq.lib()

    def apply(plan=None, n_proj=1, pools=None, rank=16, d_in=256, X=FAKE, ldx=256, y0=FAKE, ldy0=64, y=FAKE, ldy=64,
              dt=1, t=0, ws=FAKE, ws_bytes=BIG):
        plan = plan or _plan()
        pools = pools or _pool()
        return Lib.bsq_adapters_apply(ct.byref(plan), n_proj, pools, rank, d_in, _p(X), ldx, _arr(y0), _i64(ldy0),
                                      _arr(y), _i64(ldy), dt, _arr(t) if t else None, _p(ws), ws_bytes, None)
    assert apply(plan=_plan(buf=0)) == bsq.BSQ_ERR_ARG
    assert apply(plan=_plan(ids=0)) == bsq.BSQ_ERR_ARG
    assert apply(plan=_plan(M=100, buf=0), ws_bytes=0) == bsq.BSQ_ERR_BUFFER_TOO_SMALL  # no buffer needed
    assert apply(plan=_plan(M=0)) == bsq.BSQ_ERR_SHAPE
    assert apply(n_proj=0) == bsq.BSQ_ERR_ARG
    assert apply(n_proj=9) == bsq.BSQ_ERR_ARG
    assert apply(rank=0) == bsq.BSQ_ERR_ARG
    assert apply(rank=129) == bsq.BSQ_ERR_ARG
    assert apply(d_in=0) == bsq.BSQ_ERR_SHAPE
    assert apply(ldx=255) == bsq.BSQ_ERR_SHAPE
    assert apply(X=0) == bsq.BSQ_ERR_ARG
    assert apply(X=FAKE + 1) == bsq.BSQ_ERR_ALIGN
    assert apply(pools=_pool(A=0)) == bsq.BSQ_ERR_ARG
    assert apply(pools=_pool(Bp=0)) == bsq.BSQ_ERR_ARG
    assert apply(pools=_pool(d_out=0)) == bsq.BSQ_ERR_SHAPE
    assert apply(pools=_pool(scale=FAKE + 2)) == bsq.BSQ_ERR_ALIGN
    assert apply(pools=_pool(ranks=FAKE + 2)) == bsq.BSQ_ERR_ALIGN
    assert apply(y=0) == bsq.BSQ_ERR_ARG
    assert apply(ldy=63) == bsq.BSQ_ERR_SHAPE
    assert apply(ldy0=63) == bsq.BSQ_ERR_SHAPE
    assert apply(ldy0=65) == bsq.BSQ_ERR_ARG             # in place takes one stride
    assert apply(dt=2) == bsq.BSQ_ERR_DTYPE
    assert apply(y0=FAKE + 256, y=FAKE + 2, dt=0) == bsq.BSQ_ERR_ALIGN
    assert apply(y0=FAKE + 3) == bsq.BSQ_ERR_ALIGN
    assert apply(t=FAKE + 2) == bsq.BSQ_ERR_ALIGN
    assert apply(ws=0) == bsq.BSQ_ERR_ARG
    assert apply(ws=FAKE + 128) == bsq.BSQ_ERR_ALIGN
    assert apply(ws_bytes=bsq.bsq_adapters_workspace_bytes(False, 1000, 4, 16, 256, [64]) - 1) == bsq.BSQ_ERR_BUFFER_TOO_SMALL


def test_adapters_grad_rejects_before_launch():
    Lib = bsq.lib()

    def grad(plan=None, n_proj=1, pools=None, rank=16, d_in=256, X=FAKE, ldx=256, t=FAKE, dy=FAKE, lddy=64, dx0=0,
             lddx0=256, dx=FAKE, lddx=256, dt=1, dA=FAKE, dB=FAKE, acc=0, ws=FAKE, ws_bytes=BIG):
        plan = plan or _plan()
        pools = pools or _pool()
        return Lib.bsq_adapters_grad(ct.byref(plan), n_proj, pools, rank, d_in, _p(X), ldx, _arr(t), _arr(dy),
                                     _i64(lddy), _p(dx0), lddx0, _p(dx), lddx, dt, _arr(dA), _arr(dB), acc, _p(ws),
                                     ws_bytes, None)
    assert grad(t=0) == bsq.BSQ_ERR_ARG
    assert grad(dy=0) == bsq.BSQ_ERR_ARG
    assert grad(dA=0) == bsq.BSQ_ERR_ARG
    assert grad(dB=0) == bsq.BSQ_ERR_ARG
    assert grad(acc=2) == bsq.BSQ_ERR_ARG
    assert grad(lddy=63) == bsq.BSQ_ERR_SHAPE
    assert grad(lddx=255) == bsq.BSQ_ERR_SHAPE
    assert grad(dx0=FAKE + 64, lddx0=255) == bsq.BSQ_ERR_SHAPE
    assert grad(dx0=FAKE, lddx0=264) == bsq.BSQ_ERR_ARG  # in place takes one stride
    assert grad(dx0=FAKE, dt=0) == bsq.BSQ_ERR_ARG       # and one type
    assert grad(dt=3) == bsq.BSQ_ERR_DTYPE
    assert grad(dx=FAKE + 2, dt=0) == bsq.BSQ_ERR_ALIGN
    assert grad(t=FAKE + 2) == bsq.BSQ_ERR_ALIGN
    assert grad(dy=FAKE + 1) == bsq.BSQ_ERR_ALIGN
    assert grad(dA=FAKE + 2) == bsq.BSQ_ERR_ALIGN
    assert grad(dB=FAKE + 2) == bsq.BSQ_ERR_ALIGN
    assert grad(rank=0) == bsq.BSQ_ERR_ARG
    assert grad(ws_bytes=bsq.bsq_adapters_workspace_bytes(True, 1000, 4, 16, 256, [64]) - 1) == bsq.BSQ_ERR_BUFFER_TOO_SMALL
    # nothing of dx is looked at where it is not wanted
    assert grad(dx=0, dt=9, lddx=0, ws=0) == bsq.BSQ_ERR_ARG


# ---------------------------------------------------------------- cross entropy
@pytest.mark.parametrize("grad", [False, True])
def test_xent_workspace(grad):
    assert bsq.bsq_xent_workspace_bytes(grad, 0, 1, 8) > 0
    whole = bsq.bsq_xent_workspace_bytes(grad, 4096, 151936, 4096)
    assert whole < 4096 * 151936 * 2        # less than the logits in bf16
    for dims, status in (((-1, 1, 8), bsq.BSQ_ERR_SHAPE), ((1, 0, 8), bsq.BSQ_ERR_SHAPE), ((1, 1, 0), bsq.BSQ_ERR_SHAPE),
                         ((1, 1, 12), bsq.BSQ_ERR_SHAPE), (((1 << 20) + 1, 1, 8), bsq.BSQ_ERR_UNSUPPORTED),
                         ((1, 1 << 31, 8), bsq.BSQ_ERR_UNSUPPORTED), ((1, 1, 1 << 17), bsq.BSQ_ERR_UNSUPPORTED)):
        with pytest.raises(bsq.BsqError) as e:
            bsq.bsq_xent_workspace_bytes(grad, *dims)
        assert e.value.status == status, dims


def test_xent_rejects_before_launch():
    Lib = bsq.lib()

    def call(grad, H=FAKE, ldh=64, V=FAKE, ldv=64, T=10, N=100, D=64, target=FAKE, a=FAKE, b=FAKE, dH=FAKE, lddh=64,
             dV=FAKE, lddv=64, dt=1, acc=0, err=0, ws=FAKE, ws_bytes=BIG):
        if not grad:
            return Lib.bsq_xent_loss(_p(H), ldh, _p(V), ldv, T, N, D, _p(target), _p(a), _p(b), _p(err), _p(ws),
                                     ws_bytes, None)
        return Lib.bsq_xent_grad(_p(H), ldh, _p(V), ldv, T, N, D, _p(target), _p(a), _p(b), _p(dH), lddh, _p(dV),
                                 lddv, dt, acc, _p(err), _p(ws), ws_bytes, None)
    for g in (False, True):
        assert call(g, H=0) == bsq.BSQ_ERR_ARG
        assert call(g, V=0) == bsq.BSQ_ERR_ARG
        assert call(g, target=0) == bsq.BSQ_ERR_ARG
        assert call(g, a=0) == bsq.BSQ_ERR_ARG
        assert call(g, b=0) == bsq.BSQ_ERR_ARG
        assert call(g, ws=0) == bsq.BSQ_ERR_ARG
        assert call(g, T=-1) == bsq.BSQ_ERR_SHAPE
        assert call(g, N=0) == bsq.BSQ_ERR_SHAPE
        assert call(g, D=60) == bsq.BSQ_ERR_SHAPE            # not a multiple of 8
        assert call(g, ldh=63) == bsq.BSQ_ERR_SHAPE
        assert call(g, ldv=63) == bsq.BSQ_ERR_SHAPE
        assert call(g, ldv=68) == bsq.BSQ_ERR_SHAPE
        assert call(g, H=FAKE + 1) == bsq.BSQ_ERR_ALIGN
        assert call(g, V=FAKE + 8) == bsq.BSQ_ERR_ALIGN
        assert call(g, target=FAKE + 4) == bsq.BSQ_ERR_ALIGN
        assert call(g, a=FAKE + 2) == bsq.BSQ_ERR_ALIGN
        assert call(g, b=FAKE + 2) == bsq.BSQ_ERR_ALIGN
        assert call(g, err=FAKE + 2) == bsq.BSQ_ERR_ALIGN
        assert call(g, ws=FAKE + 64) == bsq.BSQ_ERR_ALIGN
        assert call(g, ws_bytes=bsq.bsq_xent_workspace_bytes(g, 10, 100, 64) - 1) == bsq.BSQ_ERR_BUFFER_TOO_SMALL
    assert call(True, dH=0) == bsq.BSQ_ERR_ARG
    assert call(True, lddh=63) == bsq.BSQ_ERR_SHAPE
    assert call(True, lddv=63) == bsq.BSQ_ERR_SHAPE
    assert call(True, dt=5) == bsq.BSQ_ERR_DTYPE
    assert call(True, acc=-1) == bsq.BSQ_ERR_ARG
    assert call(True, dV=FAKE + 2, dt=0) == bsq.BSQ_ERR_ALIGN


# ---------------------------------------------------------------- clipping
def test_clip_rejects_before_launch():
    Lib = bsq.lib()
    need = ct.c_size_t(0)
    assert Lib.bsq_clip_table_bytes(2, _i64(10, 1 << 33), ct.byref(need)) == bsq.BSQ_OK and need.value > 0
    assert Lib.bsq_clip_table_bytes(2, _i64(10, -1), ct.byref(need)) == bsq.BSQ_ERR_SHAPE
    assert Lib.bsq_clip_table_bytes(0, _i64(10), ct.byref(need)) == bsq.BSQ_ERR_ARG
    assert Lib.bsq_clip_table_bytes(1, None, ct.byref(need)) == bsq.BSQ_ERR_ARG
    assert Lib.bsq_clip_table_bytes(1, _i64(10), None) == bsq.BSQ_ERR_ARG
    assert Lib.bsq_clip_table_bytes(1, _i64(1 << 43), ct.byref(need)) == bsq.BSQ_ERR_UNSUPPORTED

    def prepare(table=FAKE, count=1, nbytes=BIG, src=FAKE, dst=None, size=100, dt=0):
        plan = B.bsq_clip_plan(table or None, count, 0)
        return Lib.bsq_clip_prepare(ct.byref(plan), nbytes, _arr(src), None if dst is None else _arr(dst), _i64(size),
                                    (ct.c_int32 * 1)(dt), None)
    assert prepare(table=0) == bsq.BSQ_ERR_ARG
    assert prepare(table=FAKE + 16) == bsq.BSQ_ERR_ALIGN
    assert prepare(count=0) == bsq.BSQ_ERR_ARG
    assert prepare(src=0) == bsq.BSQ_ERR_ARG
    assert prepare(dst=0) == bsq.BSQ_ERR_ARG
    assert prepare(dt=2) == bsq.BSQ_ERR_DTYPE
    assert prepare(src=FAKE + 2) == bsq.BSQ_ERR_ALIGN
    assert prepare(src=FAKE + 2, dst=FAKE + 1, dt=1) == bsq.BSQ_ERR_ALIGN
    assert prepare(size=-5) == bsq.BSQ_ERR_SHAPE
    assert prepare(nbytes=64) == bsq.BSQ_ERR_BUFFER_TOO_SMALL
    for fn in (Lib.bsq_grad_norm, Lib.bsq_grad_clip):
        def clip(table=FAKE, count=1, chunks=1, m=1.0, stats=FAKE, err=0):
            plan = B.bsq_clip_plan(table or None, count, chunks)
            return fn(ct.byref(plan), m, _p(stats), _p(err), None)
        assert clip(table=0) == bsq.BSQ_ERR_ARG
        assert clip(count=0) == bsq.BSQ_ERR_ARG
        assert clip(chunks=-1) == bsq.BSQ_ERR_ARG
        assert clip(m=-1.0) == bsq.BSQ_ERR_ARG
        assert clip(m=float("nan")) == bsq.BSQ_ERR_ARG
        assert clip(stats=0) == bsq.BSQ_ERR_ARG
        assert clip(stats=FAKE + 2) == bsq.BSQ_ERR_ALIGN
        assert clip(err=FAKE + 2) == bsq.BSQ_ERR_ALIGN
        assert clip(table=FAKE + 8) == bsq.BSQ_ERR_ALIGN


# ---------------------------------------------------------------- the binding's own checks
def test_binding_refuses_host_tensors_and_wrong_shapes():
    z = lambda *s, dt=torch.bfloat16: torch.zeros(s, dtype=dt)  # noqa: E731
    with pytest.raises(ValueError, match="GPU"):
        bsq.AdapterPool(z(2, 16, 64), z(2, 32, 16))
    with pytest.raises(TypeError, match="A"):
        bsq.AdapterPool(z(2, 16, 64, dt=torch.float32), z(2, 32, 16))
    with pytest.raises(ValueError, match="B"):
        bsq.AdapterPool(z(2, 16, 64), z(2, 32, 8))
    with pytest.raises(ValueError, match="3|must be"):
        bsq.AdapterPool(z(16, 64), z(32, 16))
    with pytest.raises(TypeError, match="scale"):
        bsq.AdapterPool(z(2, 16, 64), z(2, 32, 16), scale=z(2))
    with pytest.raises(ValueError, match="GPU"):
        bsq.bsq_adapters_plan(torch.zeros(4, dtype=torch.int32), 2)
    t = torch.zeros(4, dtype=torch.int64)
    with pytest.raises(ValueError, match="GPU"):
        bsq.bsq_xent_loss(z(4, 64), z(10, 64), t)
    with pytest.raises(TypeError, match="target"):
        bsq.bsq_xent_loss(z(4, 64), z(10, 64), t.int())
    with pytest.raises(ValueError, match="V"):
        bsq.bsq_xent_loss(z(4, 64), z(10, 72), t)
    with pytest.raises(TypeError, match="H"):
        bsq.bsq_xent_loss(z(4, 64, dt=torch.float32), z(10, 64), t)
    with pytest.raises(ValueError, match="contiguous"):
        bsq.bsq_xent_loss(z(64, 4).T, z(10, 64), t)
    f = torch.zeros(4)
    with pytest.raises(ValueError, match="accumulate"):
        bsq.bsq_xent_grad(z(4, 64), z(10, 64), t, f, f, accumulate=True)
    with pytest.raises(ValueError, match="no tensors"):
        bsq.GradPlan([])
    with pytest.raises(ValueError, match="GPU"):
        bsq.GradPlan([f])
    with pytest.raises(ValueError, match="contiguous"):
        bsq.GradPlan([torch.zeros(4, 4).T])
    with pytest.raises(ValueError, match="output"):
        bsq.GradPlan([f], [f, f])
