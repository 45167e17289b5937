"""Adapters of many requests (bsq_adapters_plan, bsq_adapters_apply,
bsq_adapters_grad) against the formulas in fp64:
  t = A x, y = y0 + s B t, u = s B^T dy, dx = dx0 + sum A^T u,
  dA = sum u x^T, dB = s sum dy t^T, over each adapter's tokens.

Bars, per output, from the kernels' arithmetic (products of bf16 are exact in
fp32). A sum of n products on the matrix cores rounds at least after every
four of them: at most gamma(n) = (n / 4 + 16) 2^-24 of the sum of magnitudes
(the 16 covers the split sums and the additions after them). t and u enter
their second product as two bf16 parts for bf16 results (2^-16 of each value is
lost) and as three for fp32 ones (2^-23 with the rounding of s t). The result is
rounded once: 2^-8 (bf16) or 2^-24 (fp32) of its magnitude.
"""
import math

import pytest
import torch

import paper_2607_08643_amd as bsq
from parity_bounds import say

pytestmark = pytest.mark.gpu

U32 = 2.0 ** -24
U16 = 2.0 ** -8
NONE = -1


def gamma(n):
    return (n / 4 + 16) * U32


def _ids(kind, M, n, seed):
    g = torch.Generator().manual_seed(seed)
    if kind == "none":
        return torch.full((M,), NONE, dtype=torch.int32)
    if kind == "one":
        return torch.full((M,), n - 1, dtype=torch.int32)
    if kind == "runs":
        cuts = torch.sort(torch.randint(0, M, (n,), generator=g)).values
        ids = torch.bucketize(torch.arange(M), cuts) % n
        ids[: M // 7] = NONE
        return ids.int()
    ids = torch.randint(-1, n, (M,), generator=g)  # each its own, some none
    return ids.int()


def _strided(t, pad, gpu, offset=0):
    """t on the GPU in rows `pad` elements apart beyond its width, from an
    element offset on; what lies between is NaN."""
    rows, cols = t.shape
    buf = torch.full((rows * (cols + pad) + offset,), float("nan"), dtype=t.dtype, device=gpu)
    v = buf[offset:].view(rows, cols + pad)[:, :cols] if pad else buf[offset:].view(rows, cols)
    v.copy_(t)
    return v


class Batch:
    def __init__(self, gpu, M, dims, d_in, rank, n, ids, ranks=None, y_dtype=torch.bfloat16, pad=0, offset=0, seed=1,
                 scaled=True):
        g = torch.Generator().manual_seed(seed)
        rn = lambda *s: torch.randn(s, generator=g)  # noqa: E731
        self.M, self.dims, self.d_in, self.rank, self.n = M, dims, d_in, rank, n
        self.ids = ids.to(gpu)
        self.X = _strided(rn(M, d_in).bfloat16(), pad, gpu, offset)
        self.r = [rank] * n if ranks is None else ranks
        rt = None if ranks is None else torch.tensor(ranks, dtype=torch.int32, device=gpu)
        self.pools = []
        for d_out in dims:
            A = (rn(n, rank, d_in) / math.sqrt(d_in)).bfloat16()
            B = rn(n, d_out, rank).mul(0.3).bfloat16()
            for a in range(n):  # past an adapter's rank: anything
                A[a, max(0, self.r[a]):] = float("nan")
                B[a, :, max(0, self.r[a]):] = float("nan")
            scale = torch.rand(n, generator=g) + 0.5 if scaled else None
            self.pools.append(bsq.AdapterPool(A.to(gpu), B.to(gpu), None if scale is None else scale.to(gpu), rt))
        self.base = [_strided(rn(M, d).to(y_dtype), pad, gpu, offset) for d in dims]
        self.y_dtype = y_dtype

    def adapter(self, p, a):
        """A, B (fp64, within the rank), s of adapter a of projection p."""
        q, r = self.pools[p], max(0, min(self.r[a], self.rank))
        s = 1.0 if q.scale is None else float(q.scale[a])
        return q.A[a, :r].double(), q.B[a, :, :r].double(), s, r

    def tokens(self, a):
        return (self.ids == a).nonzero()[:, 0]


def _round_bar(y, dtype):
    return (U16 if dtype == torch.bfloat16 else U32) * y.abs()


def _assert_close(got, want, tol, what):
    assert got.shape == want.shape, what
    err = (got.double() - want).abs()
    assert not torch.isnan(got.double()).any(), what
    worst = float((err / tol.clamp_min(1e-300)).max()) if err.numel() else 0.0
    say(f"  {what}: worst err/tol {worst:.3f}")
    assert (err <= tol).all(), what


def _check_apply(b, y, t, base):
    lost = 2.0 ** -16 if b.y_dtype == torch.bfloat16 else 2.0 ** -23
    for p, d_out in enumerate(b.dims):
        want = torch.zeros((b.M, d_out), dtype=torch.float64, device=y[p].device) if base is None else base[p].double()
        tol = torch.zeros_like(want)
        want_t = torch.zeros((b.M, b.rank), dtype=torch.float64, device=y[p].device)
        tol_t = torch.zeros_like(want_t)
        for a in range(b.n):
            m = b.tokens(a)
            A, B, s, r = b.adapter(p, a)
            x = b.X[m].double()
            tt = x @ A.T
            et = gamma(b.d_in) * (x.abs() @ A.abs().T)
            want_t[m, :r], tol_t[m, :r] = tt, et
            want[m] += s * (tt @ B.T)
            tol[m] += s * ((et + (lost + gamma(3 * b.rank)) * tt.abs()) @ B.abs().T)
        tol += _round_bar(want, b.y_dtype) + U32 * want.abs() + 1e-30
        _assert_close(y[p], want, tol * 1.01, f"y[{p}]")
        if t is not None:
            _assert_close(t[p], want_t, tol_t + 1e-30, f"t[{p}]")


CASES = [
    # M, d_out of the group, d_in, rank, n, ids, ranks, y, row padding, element offset
    (1, (64,), 256, 16, 3, "one", None, torch.bfloat16, 0, 0),
    (1, (4096, 1024, 1024), 4096, 16, 8, "mixed", None, torch.bfloat16, 0, 0),
    (1, (17,), 8, 1, 1, "none", None, torch.float32, 0, 0),
    (5, (1,), 1, 1, 2, "mixed", None, torch.float32, 0, 0),
    (16, (256,), 512, 8, 1, "one", None, torch.float32, 8, 0),
    (17, (256,), 512, 8, 2, "one", None, torch.bfloat16, 8, 8),
    (64, (333, 65), 296, 16, 64, "mixed", None, torch.bfloat16, 0, 0),
    (64, (512,), 1000, 24, 5, "mixed", "mixed", torch.float32, 8, 0),
    (100, (130,), 77, 5, 7, "mixed", "mixed", torch.bfloat16, 3, 1),
    (200, (96, 1, 257), 2048, 128, 3, "runs", "mixed", torch.float32, 0, 0),
    (333, (333,), 296, 48, 33, "mixed", None, torch.bfloat16, 0, 3),
    (1024, (320,), 264, 16, 1024, "mixed", None, torch.bfloat16, 0, 0),
    (1025, (320,), 264, 16, 4, "runs", None, torch.bfloat16, 0, 0),
    (1025, (70,), 33, 64, 4, "mixed", "mixed", torch.float32, 1, 0),
    (2500, (520, 72), 768, 32, 6, "runs", None, torch.bfloat16, 8, 0),
    (3000, (128,), 256, 16, 2, "one", None, torch.float32, 0, 0),
    (2049, (64,), 128, 16, 5, "none", None, torch.bfloat16, 0, 0),
]


def _ranks(kind, rank, n):
    return None if kind is None else [(rank * (i % 4)) // 3 for i in range(n)]  # 0, a third, two, all


def _batch(gpu, case, seed=1, **kw):
    M, dims, d_in, rank, n, ids, ranks, y, pad, offset = case
    return Batch(gpu, M, dims, d_in, rank, n, _ids(ids, M, n, seed + 3), _ranks(ranks, rank, n), y, pad, offset, seed, **kw)


@pytest.mark.parametrize("case", CASES, ids=lambda c: f"M{c[0]}-{c[1]}x{c[2]}-r{c[3]}-n{c[4]}-{c[5]}")
def test_apply_matches_formula(case, gpu):
    say(f"adapters apply {case}")
    b = _batch(gpu, case)
    plan = bsq.bsq_adapters_plan(b.ids, b.n)
    y, t = bsq.bsq_adapters_apply(plan, b.pools, b.X, b.base, keep=True)
    torch.cuda.synchronize()
    _check_apply(b, y, t, b.base)
    # without a base; in place, where rows without an adapter keep their bits
    z, none = bsq.bsq_adapters_apply(plan, b.pools, b.X, None, y_dtype=b.y_dtype)
    assert none is None
    _check_apply(b, z, None, None)
    own = [q.clone(memory_format=torch.preserve_format) for q in b.base]
    bsq.bsq_adapters_apply(plan, b.pools, b.X, own, out=own)
    torch.cuda.synchronize()
    free = (b.ids < 0)
    for o, q, w in zip(own, y, b.base):
        assert torch.equal(o, q)
        assert torch.equal(o[free], w[free])


@pytest.mark.parametrize("M,n,kind", [(257, 1, "one"), (300, 3, "mixed"), (1000, 1024, "mixed"), (1025, 7, "runs"),
                                      (5000, 40, "mixed"), (8192, 2, "none")])
def test_plan_is_a_stable_sort(M, n, kind, gpu):
    say(f"adapters plan M={M} n={n} {kind}")
    ids = _ids(kind, M, n, 5)
    plan = bsq.bsq_adapters_plan(ids.to(gpu), n)
    torch.cuda.synchronize()
    words = plan.buf.view(torch.int32).cpu()
    tile = 16 if M <= 1024 else 64
    key = torch.where(ids < 0, n, ids).long()
    want = torch.sort(key, stable=True).indices
    at = 16 + (2 * (n + 2) + 3) // 4 * 4
    assert torch.equal(words[at:at + M].long(), want)
    counts = torch.bincount(key, minlength=n + 1)
    tiles = (counts + tile - 1) // tile
    assert int(words[0]) == int(tiles[:n].sum()) and int(words[1]) == int(tiles.sum())


@pytest.mark.parametrize("M,n,kind", [(300, 64, "mixed"), (8192, 64, "runs"), (8193, 65, "mixed"), (8256, 1024, "mixed"),
                                      (20001, 5, "runs"), (70000, 1, "one")])
def test_plan_lists_every_tile_and_piece(M, n, kind, gpu):
    """Either side of 8192 tokens (up to which ids are read once) and of 64
    adapters (up to which a wave writes an adapter's tiles): the whole plan."""
    say(f"adapters plan M={M} n={n} {kind}")
    ids = _ids(kind, M, n, 11)
    plan = bsq.bsq_adapters_plan(ids.to(gpu), n)
    torch.cuda.synchronize()
    words = plan.buf.view(torch.int32).cpu().long()
    key = torch.where(ids < 0, n, ids).long()
    counts = torch.bincount(key, minlength=n + 1).tolist()
    tile, piece = 16 if M <= 1024 else 64, max(256, (M // 16 + 63) // 64 * 64)
    order = 16 + (2 * (n + 2) + 3) // 4 * 4
    assert torch.equal(words[order:order + M], torch.sort(key, stable=True).indices)
    tiles, pieces, first, slot = [], [], 0, 0
    for a, c in enumerate(counts):
        tiles += [[a if a < n else -1, first + q, min(tile, c - q), 0] for q in range(0, c, tile)]
        if a < n:
            many = c > piece
            for q in range(0, c, piece):
                pieces.append([a, first + q, min(piece, c - q), slot if many else -1])
                slot += many
        first += c
    live = sum(t[0] >= 0 for t in tiles)
    assert words[:3].tolist() == [live, len(tiles), len(pieces)]
    at = order + (M + 3) // 4 * 4
    assert words[at:at + 4 * len(tiles)].view(-1, 4).tolist() == tiles
    at += 4 * min(M, M // tile + n + 1)
    assert words[at:at + 4 * len(pieces)].view(-1, 4).tolist() == pieces


def test_an_id_out_of_range_is_reported_and_means_none(gpu):
    b = Batch(gpu, 40, (64,), 128, 16, 4, _ids("mixed", 40, 4, 9))
    ids = b.ids.clone()
    ids[[3, 17]] = torch.tensor([4, 1 << 30], dtype=torch.int32, device=gpu)
    err = torch.zeros(1, dtype=torch.int32, device=gpu)
    plan = bsq.bsq_adapters_plan(ids, 4, err=err)
    y, _ = bsq.bsq_adapters_apply(plan, b.pools, b.X, b.base)
    torch.cuda.synchronize()
    assert int(err.item()) == bsq.DEVERR_BAD_SET
    b.ids = torch.where(ids >= 4, NONE, ids)
    _check_apply(b, y, None, b.base)
    err.zero_()
    bsq.bsq_adapters_plan(b.ids, 4, err=err)
    torch.cuda.synchronize()
    assert int(err.item()) == 0


@pytest.mark.parametrize("M", [40, 1500])
def test_a_token_that_is_not_finite_stays_alone(M, gpu):
    """A NaN or infinite x (or y0) changes its own row of y and no other's."""
    b = Batch(gpu, M, (96,), 264, 16, 3, _ids("runs", M, 3, 2))
    plan = bsq.bsq_adapters_plan(b.ids, b.n)
    y, _ = bsq.bsq_adapters_apply(plan, b.pools, b.X, b.base)
    X2 = b.X.clone()
    X2[M // 2, 5], X2[M - 1, 0] = float("nan"), float("inf")
    z, _ = bsq.bsq_adapters_apply(plan, b.pools, X2, b.base)
    torch.cuda.synchronize()
    same = torch.ones(M, dtype=torch.bool)
    same[[M // 2, M - 1]] = False
    assert torch.equal(z[0][same], y[0][same])
    assert torch.isnan(z[0][M // 2]).all() and not torch.isfinite(z[0][M - 1]).all()


# ---------------------------------------------------------------- gradients
def _check_grad(b, t, dy, base, dx, dA, dB, dx_dtype, before=None):
    lost_x = 2.0 ** -16 if dx_dtype == torch.bfloat16 else 2.0 ** -23
    if dx is not None:
        want_x = torch.zeros((b.M, b.d_in), dtype=torch.float64, device=dx.device) if base is None else base.double()
        tol_x = torch.zeros_like(want_x)
    for p, d_out in enumerate(b.dims):
        for a in range(b.n):
            m = b.tokens(a)
            A, B, s, r = b.adapter(p, a)
            x, g, tt = b.X[m].double(), dy[p][m].double(), t[p][m, :r].double()
            u, eu = s * (g @ B), s * gamma(d_out) * (g.abs() @ B.abs())
            wa = torch.zeros((b.rank, b.d_in), dtype=torch.float64, device=x.device)
            wb = torch.zeros((d_out, b.rank), dtype=torch.float64, device=x.device)
            ta, tb = torch.full_like(wa, 1e-30), torch.full_like(wb, 1e-30)
            few = 2.0 ** -22 + gamma(3 * len(m))
            wa[:r] = u.T @ x
            ta[:r] += (eu + few * u.abs()).T @ x.abs()
            wb[:, :r] = s * (g.T @ tt)
            tb[:, :r] += few * s * (g.abs().T @ tt.abs())
            if before is not None:
                wa += before[0][p][a].double()
                wb += before[1][p][a].double()
                ta += U32 * wa.abs()
                tb += U32 * wb.abs()
            _assert_quiet(dA[p][a], wa, ta, f"dA[{p}][{a}]")
            _assert_quiet(dB[p][a], wb, tb, f"dB[{p}][{a}]")
            if dx is not None:
                want_x[m] += u @ A
                tol_x[m] += (eu + (lost_x + gamma(3 * b.rank * len(b.dims))) * u.abs()) @ A.abs()
    if dx is not None:
        tol_x += _round_bar(want_x, dx_dtype) + U32 * want_x.abs() + 1e-30
        _assert_close(dx, want_x, tol_x * 1.01, "dx")


def _assert_quiet(got, want, tol, what):
    err = (got.double() - want).abs()
    assert (err <= tol).all(), f"{what}: worst err/tol {float((err / tol).max()):.3f}"


@pytest.mark.parametrize("case", CASES, ids=lambda c: f"M{c[0]}-{c[1]}x{c[2]}-r{c[3]}-n{c[4]}-{c[5]}")
def test_gradients_match_formula(case, gpu):
    say(f"adapters grad {case}")
    b = _batch(gpu, case, seed=2)
    pad, offset = case[8], case[9]
    plan = bsq.bsq_adapters_plan(b.ids, b.n)
    _, t = bsq.bsq_adapters_apply(plan, b.pools, b.X, None, keep=True)
    for p in range(len(t)):  # past an adapter's rank: not used
        for a in range(b.n):
            t[p][b.tokens(a), max(0, b.r[a]):] = float("nan")
    g = torch.Generator().manual_seed(8)
    dy = [_strided(torch.randn((b.M, d), generator=g).bfloat16(), pad, gpu, offset) for d in b.dims]
    base = _strided(torch.randn((b.M, b.d_in), generator=g).bfloat16(), pad, gpu, offset)
    dx, dA, dB = bsq.bsq_adapters_grad(plan, b.pools, b.X, t, dy, base=base)
    torch.cuda.synchronize()
    _check_grad(b, t, dy, base, dx, dA, dB, torch.bfloat16)
    # no base, 32-bit dx, added to what is there
    before = ([torch.randn_like(q) for q in dA], [torch.randn_like(q) for q in dB])
    grads = ([q.clone() for q in before[0]], [q.clone() for q in before[1]])
    dx, dA2, dB2 = bsq.bsq_adapters_grad(plan, b.pools, b.X, t, dy, dx_dtype=torch.float32, grads=grads, accumulate=True)
    torch.cuda.synchronize()
    assert dA2[0] is grads[0][0] and dB2[-1] is grads[1][-1]
    _check_grad(b, t, dy, None, dx, dA2, dB2, torch.float32, before)
    # dx in place; without dx
    own = base.clone(memory_format=torch.preserve_format)
    first, dA3, _ = bsq.bsq_adapters_grad(plan, b.pools, b.X, t, dy, base=own, dx=own)
    none, dA4, dB4 = bsq.bsq_adapters_grad(plan, b.pools, b.X, t, dy, want_dx=False)
    torch.cuda.synchronize()
    assert first is own and none is None
    for q, w in zip(dA3 + dA4 + dB4, dA + dA + dB):
        assert torch.equal(q, w)


def test_gradients_match_differences(gpu):
    """y is linear in A, in B and in x, so the change of <w, y> under a change of
    one of them is the gradient's product with that change, exactly. Values on
    a coarse grid keep both ends exact in bf16; what is left are the fp32 sums of y
    (gamma of the depth) and of the gradients."""
    M, d_out, d_in, rank, n = 300, 200, 120, 16, 3
    g = torch.Generator().manual_seed(4)
    grid = lambda *s: (torch.randint(-8, 9, s, generator=g) / 16).bfloat16().to(gpu)  # noqa: E731
    ids = _ids("mixed", M, n, 6).to(gpu)
    A, B, X, w = grid(n, rank, d_in), grid(n, d_out, rank), grid(M, d_in), grid(M, d_out)
    scale = torch.tensor([1.0, 0.5, 2.0], device=gpu)
    plan = bsq.bsq_adapters_plan(ids, n)

    def value(A, B, X):
        y, _ = bsq.bsq_adapters_apply(plan, bsq.AdapterPool(A, B, scale), X, None, y_dtype=torch.float32)
        return float((y.double() * w.double()).sum())

    pool = bsq.AdapterPool(A, B, scale)
    _, t = bsq.bsq_adapters_apply(plan, pool, X, None, keep=True)
    dx, dA, dB = bsq.bsq_adapters_grad(plan, pool, X, t, w, dx_dtype=torch.float32)
    mag = float((X.double().abs().sum(1).max() * rank * 2) * w.double().abs().sum())
    for name, q, d in (("A", A, dA), ("B", B, dB), ("x", X, dx)):
        step = (torch.randint(-2, 3, q.shape, generator=g) / 16).bfloat16().to(gpu)
        hi = {"A": A, "B": B, "X": X} | ({"X": X + step} if name == "x" else {name: q + step})
        diff = value(**hi) - value(A, B, X)
        along = float((d.double() * step.double()).sum())
        say(f"  d{name}: difference {diff:.6f}, gradient {along:.6f}")
        assert abs(diff - along) <= 4 * gamma(d_in + 3 * rank) * mag / math.sqrt(M * d_out), name


def test_results_repeat_and_a_captured_step_replays(gpu):
    """The same bits from call to call, on another stream, and from a captured graph
    replayed between eager calls."""
    b = Batch(gpu, 1500, (320, 64), 264, 16, 5, _ids("mixed", 1500, 5, 3))
    g = torch.Generator().manual_seed(1)
    dy = [torch.randn((b.M, d), generator=g).bfloat16().to(gpu) for d in b.dims]

    def step(stream=None, ws=(None, None), buf=None):
        plan = bsq.bsq_adapters_plan(b.ids, b.n, buf=buf, stream=stream)
        y, t = bsq.bsq_adapters_apply(plan, b.pools, b.X, b.base, keep=True, ws=ws[0], stream=stream)
        dx, dA, dB = bsq.bsq_adapters_grad(plan, b.pools, b.X, t, dy, ws=ws[1], stream=stream)
        return y + t + [dx] + dA + dB

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
            q.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        for q, w in zip(held, want):
            assert torch.equal(q, w)
        again = step()
        torch.cuda.synchronize()
        for q, w in zip(again, want):
            assert torch.equal(q, w)
    for q, w in zip(other, want):
        assert torch.equal(q, w)


def test_rows_past_32_bit_offsets(gpu):
    """Rows 2^24 elements apart: the last ones lie past 2^32 bytes."""
    M, ld, d_in, d_out = 200, 1 << 24, 64, 48
    b = Batch(gpu, M, (d_out,), d_in, 16, 3, _ids("mixed", M, 3, 3))
    big = torch.empty(M * ld, dtype=torch.bfloat16, device=gpu)
    X, Y = big.view(M, ld)[:, :d_in], big.view(M, ld)[:, 128:128 + d_out]
    X.copy_(b.X)
    Y.copy_(b.base[0])
    plan = bsq.bsq_adapters_plan(b.ids, b.n)
    y, t = bsq.bsq_adapters_apply(plan, b.pools, b.X, b.base, keep=True)
    bsq.bsq_adapters_apply(plan, b.pools, X, [Y], out=[Y])
    dx, dA, dB = bsq.bsq_adapters_grad(plan, b.pools, b.X, t, y)
    dx2, dA2, dB2 = bsq.bsq_adapters_grad(plan, b.pools, X, t, [Y])
    torch.cuda.synchronize()
    assert torch.equal(Y, y[0]) and torch.equal(dx, dx2) and torch.equal(dA[0], dA2[0]) and torch.equal(dB[0], dB2[0])
