// Low-rank adapters of many requests beside a shared projection, and their
// gradients. For token m with adapter a (none: the base alone)
//   t = A_a x,                 y = y0 + s_a B_a t,
//   u = s_a B_a^T dy,          dx = dx0 + A_a^T u,
//   dA_a = sum_m u x^T,        dB_a = s_a sum_m dy t^T.
//
// The tokens are sorted by adapter once per batch (adapters_plan_kernel) and
// cut into tiles of one adapter. Every product is then a small dense one on
// the matrix cores, whatever the mixture of adapters:
//
//   shrink   a tile's t: d_in is split over blocks and waves, whose fp32 partial
//            sums go to the workspace;
//   parts    sums those in order (small batches: expand does);
//   expand   adds s B t to a tile's rows of y;
//   dy       of a run of one adapter's tokens (a "piece"), dB and the partial
//            sums of u from one reading of dy;
//   da, dx   dA of a piece, and A^T u added to a tile's rows of dx.
//
// Partial results of an adapter's several pieces are added in order.
//
// t and u are held in fp32 and enter the next product as bf16 parts: the value
// rounded, then what remains, rounded. For bf16 results two parts (2^-16 of the
// value is lost, and a rank block of 16 with its two parts fills one 32-deep
// product), for fp32 results three (2^-24). (An infinite entry of A or B meets all
// parts, some of them 0 or of the other sign: its results may be NaN where the
// formula's are infinite.)
#include <algorithm>
#include <type_traits>

#include "adapter_rows.h"
#include "gemm_common.h"

namespace bsq {
namespace {

constexpr int AT = 256;  // threads of a block: 4 waves

// Up to this many tokens a forward call groups them itself, every block from the
// ids: a plan's launch (5 us) would be a third of a decode step's time.
constexpr int64_t DIRECT_TOKENS = BSQ_ADAPTERS_DIRECT;
constexpr int PLAN_WAVES = 16, PLAN_AHEAD = 8;  // groups of 64 ids that a wave has in flight

struct PlanLayout {
    int64_t tile, piece;              // tokens of a tile, of a piece
    int64_t max_tiles, max_pieces, max_slots;
    int64_t seg, order, tiles, pieces, words;  // offsets and size in int32 words
};

// Header words of a plan: tiles with an adapter, all tiles, pieces.
constexpr int PLAN_HDR = 16;

PlanLayout plan_layout(int64_t M, int64_t n)
{
    PlanLayout l{};
    // Tokens of a tile: 16 leave fewer idle where adapters have few tokens each, 64
    // read an adapter's weights less often (q, k and v of 4096 inputs at rank 16, mixed
    // tokens of 64 adapters, apply: 768 tokens 27 us with 16, 30 with 64; 4096 tokens 63
    // and 53; between 1024 and 2048, and with few adapters, both are within 7%)
    l.tile = (M <= 1024) ? 16 : 64;
    l.piece = std::max<int64_t>(256, (M / 16 + 63) / 64 * 64);
    l.max_tiles = std::min(M, M / l.tile + n + 1);
    l.max_pieces = std::min(M, M / l.piece + n);
    // pieces of adapters that have several: each but the last of one is whole
    l.max_slots = std::min(l.max_pieces, 2 * (M / l.piece));
    l.seg = PLAN_HDR;                       // [n + 2]: first place of an adapter's tokens; pieces' first [n + 2] after
    l.order = l.seg + (2 * (n + 2) + 3) / 4 * 4;
    l.tiles = l.order + (M + 3) / 4 * 4;    // int4: adapter, first place, tokens, 0
    l.pieces = l.tiles + 4 * l.max_tiles;   // int4: adapter, first place, tokens, slot (-1: the adapter's only one)
    l.words = l.pieces + 4 * l.max_pieces;
    return l;
}

struct PlanArgs {
    const int32_t *ids;
    int32_t *buf, *err;
    int64_t M;
    int n, bits;  // bits: of a key 0 .. n
    PlanLayout l;
};

// Inclusive scans over the first `waves` waves' threads of four counts, and the
// counts' sums.
__device__ __forceinline__ void block_scan4(int (&v)[4], int (&all)[4], int waves, int (*s_wave)[4])
{
    const int t = threadIdx.x, lane = t & 63, w = t >> 6;
    if (w < waves) {
#pragma unroll 1
        for (int d = 1; d < 64; d <<= 1)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const int o = __shfl_up(v[q], d);
                if (lane >= d) v[q] += o;
            }
        if (lane == 63)
#pragma unroll
            for (int q = 0; q < 4; ++q) s_wave[w][q] = v[q];
    }
    __syncthreads();
#pragma unroll
    for (int q = 0; q < 4; ++q) all[q] = 0;
#pragma unroll 1
    for (int k = 0; k < waves; ++k)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            all[q] += s_wave[k][q];
            if (k < w) v[q] += s_wave[k][q];
        }
}

// A stable counting sort in one block: each wave counts a run of tokens into
// its own row of counters (lanes of equal keys are found by ballots over the
// key's bits; their first adds for all), the rows are scanned, and each wave
// goes over its run again to place its tokens. No atomics: the order, and with
// it every sum over tokens, is fixed. One compute unit issues all of it (about
// 1 us per 1024 tokens beside 4.5 us), so what the ballots find waits in LDS and
// up to 8192 tokens the second time is a lookup (8192 tokens of 4 adapters 12.0 us,
// found again 13.5).
__global__ __launch_bounds__(64 * PLAN_WAVES) void adapters_plan_kernel(const PlanArgs a)
{
    extern __shared__ int32_t s_cnt[];  // [PLAN_WAVES][n + 1]
    __shared__ int s_wave[PLAN_WAVES][4];
    __shared__ int2 s_tile[64];
    __shared__ int32_t s_ids[PLAN_WAVES][64 * PLAN_AHEAD];
    const int t = threadIdx.x, lane = t & 63, w = t >> 6, nk = a.n + 1;
    int32_t *row = s_cnt + w * nk;
    for (int k = t; k < PLAN_WAVES * nk; k += 64 * PLAN_WAVES) s_cnt[k] = 0;
    __syncthreads();
    const int M = int(a.M), per = ((M + PLAN_WAVES - 1) / PLAN_WAVES + 63) / 64 * 64;
    const int lo = w * per, hi = (lo + per < M) ? lo + per : M;
    int32_t *order = a.buf + a.l.order;
    bool bad = false;
    // PLAN_AHEAD groups of 64 ids from m1 on: each lane's key (bits 0-10), how many lanes
    // before it have the same (11-16), how many in all (17-23), and whether it has a token (24)
    auto group = [&](int m1) {
        int32_t id[PLAN_AHEAD];
#pragma unroll
        for (int q = 0; q < PLAN_AHEAD; ++q) id[q] = (m1 + 64 * q + lane < hi) ? a.ids[m1 + 64 * q + lane] : -1;
#pragma unroll
        for (int q = 0; q < PLAN_AHEAD; ++q) s_ids[w][64 * q + lane] = id[q];
#pragma unroll 1
        for (int q = 0; q < PLAN_AHEAD; ++q) {
            if (m1 + 64 * q >= hi) break;
            const int mine = s_ids[w][64 * q + lane];
            const bool in = m1 + 64 * q + lane < hi;
            bad |= mine >= a.n;
            const int key = (mine >= 0 && mine < a.n) ? mine : a.n;
            uint64_t same = __ballot(in);
#pragma unroll 1
            for (int b = 0; b < a.bits; ++b) {
                const bool one = (key >> b) & 1;
                const uint64_t ones = __ballot(one);
                const uint32_t flip = one ? 0u : ~0u;
                same &= ones ^ (uint64_t(flip) << 32 | flip);
            }
            const int before = __popcll(same & ((uint64_t(1) << lane) - 1));
            s_ids[w][64 * q + lane] = key | before << 11 | __popcll(same) << 17 | int(in) << 24;
        }
    };
    // pass 0 counts, pass 1 places
    for (int pass = 0; pass < 2; ++pass) {
        for (int m1 = lo; m1 < hi; m1 += 64 * PLAN_AHEAD) {
            if (pass == 0 || per > 64 * PLAN_AHEAD) group(m1);  // (each lane reads back what it wrote)
#pragma unroll 1
            for (int q = 0; q < PLAN_AHEAD; ++q) {
                if (m1 + 64 * q >= hi) break;
                const int e = s_ids[w][64 * q + lane], key = e & 2047, before = (e >> 11) & 63;
                const bool in = e >> 24;
                const int at = row[key];
                if (pass == 1 && in) order[at + before] = m1 + 64 * q + lane;
                // (a wave's LDS operations run in order, so the reads above come first)
                if (in && before == 0) row[key] = at + ((e >> 17) & 127);
            }
        }
        __syncthreads();
        if (pass == 1) break;
        // thread k: the counts of adapter k
        int total = 0;
        if (t < a.n)
#pragma unroll 4
            for (int v = 0; v < PLAN_WAVES; ++v) total += s_cnt[v * nk + t];
        const int T = int(a.l.tile), P = int(a.l.piece);
        auto write_tiles = [&](int ad, int start, int count, int at, int from, int step) {
            int4 *tl = reinterpret_cast<int4 *>(a.buf + a.l.tiles) + at;
#pragma unroll 1
            for (int q = from; q * T < count; q += step)
                tl[q] = make_int4(ad, start + q * T, count - q * T < T ? count - q * T : T, 0);
        };
        const int nt = (total + T - 1) / T, np = (total + P - 1) / P, ns = (np > 1) ? np : 0;
        int v[4] = {total, nt, np, ns}, all[4];
        block_scan4(v, all, (a.n + 63) / 64, s_wave);
        const int start = v[0] - total;
        if (t < a.n) {
            int at = start;
            for (int q = 0; q < PLAN_WAVES; ++q) {
                const int c = s_cnt[q * nk + t];
                s_cnt[q * nk + t] = at;
                at += c;
            }
            int32_t *seg = a.buf + a.l.seg;
            seg[t] = start;
            seg[a.n + 2 + t] = v[2] - np;
            if (a.n <= 64) s_tile[t] = make_int2(v[1] - nt, total);
            else write_tiles(t, start, total, v[1] - nt, 0, 1);
            int4 *pc = reinterpret_cast<int4 *>(a.buf + a.l.pieces) + (v[2] - np);
            for (int q = 0; q < np; ++q)
                pc[q] = make_int4(t, start + q * P, total - q * P < P ? total - q * P : P, ns ? v[3] - ns + q : -1);
        }
        // few adapters may have many tiles each: a wave writes them
        if (a.n <= 64) {
            __syncthreads();
            for (int k = w; k < a.n; k += PLAN_WAVES) write_tiles(k, s_cnt[k], s_tile[k].y, s_tile[k].x, lane, 64);
        }
        // the tokens without an adapter follow
        const int live = all[0], none = M - live, nnt = (none + T - 1) / T;
        if (t == 0) {
            int at = live;
            for (int q = 0; q < PLAN_WAVES; ++q) {
                const int c = s_cnt[q * nk + a.n];
                s_cnt[q * nk + a.n] = at;
                at += c;
            }
            int32_t *seg = a.buf + a.l.seg;
            seg[a.n] = live;
            seg[a.n + 1] = M;
            seg[a.n + 2 + a.n] = all[2];
            seg[a.n + 2 + a.n + 1] = all[2];
            a.buf[0] = all[1];
            a.buf[1] = all[1] + nnt;
            a.buf[2] = all[2];
        }
        write_tiles(-1, live, none, all[1], t, 64 * PLAN_WAVES);
        __syncthreads();
    }
    if (bad && a.err) atomicOr(a.err, BSQ_DEVERR_BAD_SET);
}

// ---------------------------------------------------------------------------
// Shared by the products. A rank is cut into blocks of 16; the blocks of all
// projections of a group are numbered through (block v: ranks 16 (v % rb) .. of
// projection v / rb).
// ---------------------------------------------------------------------------
struct Proj {
    const uint16_t *A, *B;   // [n][rank][d_in], [n][d_out][rank]
    const float *scale;      // [n] or NULL
    const int32_t *ranks;    // [n] or NULL
    const void *base;        // y0 (dy in the backward pass)
    void *y;
    float *t;                // [M][rank], token order (written forward, read backward) or NULL
    float *dA, *dB;
    int64_t d_out, ldb, ldy;
};

struct AdArgs {
    const int32_t *plan;      // (or NULL: the tokens are grouped from ids)
    const int32_t *ids;
    PlanLayout l;
    Proj p[BSQ_MAX_GROUP];
    const uint16_t *X;
    const uint16_t *dx0;
    void *dx;
    int64_t M, d_in, ldx, lddx0, lddx;
    int n, np, rank, rb, nv, ksplit, ecols;
    int accumulate;
    float *part;      // forward [ksplit][nv][M][16], backward [chunks][nv][M][16]: partial t or u
    uint16_t *hl;     // [nv][M][3][16]: s t or u as three bf16 parts
    float *slots;     // partial dB and dA
    int64_t slot_floats;
};

__device__ __forceinline__ float scale_of(const Proj &p, int a) { return p.scale ? p.scale[a] : 1.0f; }

__device__ __forceinline__ int rank_of(const Proj &p, int a, int rank)
{
    if (!p.ranks) return rank;
    const int r = p.ranks[a];
    return r < 0 ? 0 : (r < rank ? r : rank);
}

typedef u32x4_t frag_t;

__device__ __forceinline__ frag_t zero_frag() { return frag_t{0u, 0u, 0u, 0u}; }

__device__ __forceinline__ bf16x8_t as_bf16(frag_t v) { return __builtin_bit_cast(bf16x8_t, v); }

__device__ __forceinline__ f32x4_t mfma(frag_t l, frag_t r, f32x4_t c)
{
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16(l), as_bf16(r), c, 0, 0, 0);
}

// A load under a condition is waited for where it stands. So loads are
// unconditional, from where there is something to read, and what is not part of
// the data is masked where it is used. They are of 16 bytes at any alignment of
// their elements (global memory takes that; element by element, odd row lengths
// took several times as long).
typedef u32x4_t any_u32x4_t __attribute__((aligned(2)));
typedef f32x4_t any_f32x4_t __attribute__((aligned(4)));

__device__ __forceinline__ frag_t load16(const void *p) { return *static_cast<const any_u32x4_t *>(p); }

// v without its first s (0 to 7) values.
__device__ __forceinline__ frag_t drop8(frag_t v, int s)
{
    if (s & 4) v = frag_t{v[2], v[3], 0u, 0u};
    if (s & 2) v = frag_t{v[1], v[2], v[3], 0u};
    if (s & 1) v = frag_t{(v[0] >> 16) | (v[1] << 16), (v[1] >> 16) | (v[2] << 16), (v[2] >> 16) | (v[3] << 16), v[3] >> 16};
    return v;
}

// Values k .. k + 7 (k a multiple of 8) of n; those past the end are others of
// them. EVEN: n is a multiple of 8.
template <bool EVEN>
__device__ __forceinline__ frag_t raw8(const uint16_t *p, int64_t k, int64_t n)
{
    if constexpr (EVEN) return load16(p + (k < n ? k : 0));
    if (n >= 8) {
        const int64_t from = k < n - 8 ? k : n - 8;
        const frag_t v = load16(p + from);
        return drop8(v, k < n ? int(k - from) : 0);
    }
    frag_t v = zero_frag();
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e >> 1] |= uint32_t(p[k + e < n ? k + e : n - 1]) << (16 * (e & 1));
    return v;
}

// Values from `start` on of an array of n, whatever they are past a row's end.
// EVEN: rows of multiples of 8.
template <bool EVEN>
__device__ __forceinline__ frag_t flat8(const uint16_t *p, int64_t start, int64_t n)
{
    if constexpr (EVEN) return load16(p + start);
    if (n >= 8) {
        const int64_t from = start < n - 8 ? start : n - 8;
        const frag_t v = load16(p + from);
        return drop8(v, start < n ? int(start - from) : 0);
    }
    frag_t v = zero_frag();
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e >> 1] |= uint32_t(p[start + e < n ? start + e : n - 1]) << (16 * (e & 1));
    return v;
}

// v's first `left` values, zeros behind them. EVEN: all eight or none.
template <bool EVEN>
__device__ __forceinline__ frag_t first8(frag_t v, int64_t left)
{
    if constexpr (EVEN) {
        const uint32_t m = left > 0 ? ~0u : 0u;
        return frag_t{v[0] & m, v[1] & m, v[2] & m, v[3] & m};
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] &= (left > 2 * e ? 0xffffu : 0u) | (left > 2 * e + 1 ? 0xffff0000u : 0u);
    return v;
}

// The bf16 parts of x: rounded, and what remains, rounded, twice (nothing
// where the value is or has become infinite).
__device__ __forceinline__ void split3(const float (&x)[8], frag_t (&part)[3])
{
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        float a = x[2 * e], b = x[2 * e + 1];
#pragma unroll
        for (int q = 0; q < 3; ++q) {
            part[q][e] = pack_bf16x2(a, b);
            const float ha = __uint_as_float(part[q][e] << 16), hb = __uint_as_float(part[q][e] & 0xffff0000u);
            a = (ha - ha == 0.0f) ? a - ha : 0.0f;
            b = (hb - hb == 0.0f) ? b - hb : 0.0f;
        }
    }
}

// A tile as a wave sees it: the lane's token (that of a place past the tile's
// end is its last), its place in t's partial sums, and whether it is the tile's.
struct TileView {
    int adapter, count;
    int64_t token, place, first;  // first: place of the tile's first token (not DIRECT)
    bool live;
};

// DIRECT (up to DIRECT_TOKENS tokens): block b is the tile whose first token is
// b, the k-th of its adapter with k a multiple of 16; every wave finds the tile
// from the ids. Places are tokens. False: there is no such tile.
template <bool DIRECT, int TG>
__device__ __forceinline__ bool tile_view(const AdArgs &a, bool with_none, int (*s_tok)[16], TileView &v)
{
    const int t = threadIdx.x, lane = t & 63, r16 = lane & 15;
    const int wave = __builtin_amdgcn_readfirstlane(t >> 6);
    const int b = blockIdx.x;
    if constexpr (DIRECT) {
        constexpr int W = int(DIRECT_TOKENS / 64);
        int id[W];
        const int raw = a.ids[b];
        const int mine = (raw >= 0 && raw < a.n) ? raw : -1;
        if (mine < 0 && !with_none) return false;
        int before = 0, all = 0, at[W];
        bool same[W];
#pragma unroll
        for (int w = 0; w < W; ++w) id[w] = a.ids[64 * w + lane < a.M ? 64 * w + lane : 0];
#pragma unroll
        for (int w = 0; w < W; ++w) {
            same[w] = ((id[w] >= 0 && id[w] < a.n) ? id[w] : -1) == mine && 64 * w + lane < a.M;
            const uint64_t mask = __ballot(same[w]);
            at[w] = all + __popcll(mask & ((uint64_t(1) << lane) - 1));
            if ((b >> 6) == w) before = all + __popcll(mask & ((uint64_t(1) << (b & 63)) - 1));
            all += __popcll(mask);
        }
        if (before & 15) return false;
#pragma unroll
        for (int w = 0; w < W; ++w)
            if (same[w] && at[w] >= before && at[w] < before + 16) s_tok[wave][at[w] - before] = 64 * w + lane;
        v.adapter = mine;
        v.count = (all - before < 16) ? all - before : 16;
        v.live = r16 < v.count;
        __builtin_amdgcn_wave_barrier();
        v.token = v.place = s_tok[wave][v.live ? r16 : v.count - 1];
        return true;
    } else {
        if (b >= a.plan[with_none ? 1 : 0]) return false;
        const int4 tile = reinterpret_cast<const int4 *>(a.plan + a.l.tiles)[b];
        const int tok = (TG == 1 ? 0 : 16 * wave) + r16;
        v.adapter = tile.x;
        v.count = tile.z;
        v.first = tile.y;
        v.live = tok < tile.z;
        v.place = tile.y + (v.live ? tok : tile.z - 1);
        v.token = a.plan[a.l.order + v.place];
        return true;
    }
}

// ---------------------------------------------------------------------------
// shrink: part[z][v][place][r] = sum over the block's share of d_in of A[r] x,
// for VB rank blocks v at a time. 16-token tiles: the four waves share the tile
// and split d_in. 64-token tiles: 32 tokens a wave (A is read half as often as
// with 16) and two waves along d_in. Loads are a step ahead of their products.
// Bound by reading x, whose 64-byte pieces of many rows come at 2.0 to 2.2 TB/s
// (2000 tokens of 25600 inputs at rank 64: 52 us; 8192 of 4096 for three projections
// of rank 16: 32 us).
// ---------------------------------------------------------------------------
template <int VB, bool EVEN, int TG, bool DIRECT>
__global__ __launch_bounds__(AT) void adapters_shrink(const AdArgs a)
{
    constexpr int U = 4;                        // 32-deep steps whose loads are in flight together
    constexpr int MT = (TG == 1) ? 1 : 2;       // 16-token groups of a wave
    constexpr int KW = (TG == 1) ? 4 : 2;       // waves along d_in
    __shared__ int s_tok[4][16];
    __shared__ f32x4_t s_acc[4][MT * VB][64];
    TileView tv;
    if (!tile_view<DIRECT, TG>(a, false, s_tok, tv)) return;
    const int t = threadIdx.x, lane = t & 63, g = lane >> 4, r16 = lane & 15;
    const int wave = __builtin_amdgcn_readfirstlane(t >> 6);
    const int64_t K = a.d_in;
    const int v0 = int(blockIdx.z) * VB;
    // the block's range of k, in whole turns of U steps of 32 for each wave along it,
    // and the wave's tokens
    const int kw = (TG == 1) ? wave : wave & 1, tg = (TG == 1) ? 0 : wave >> 1;
    const int64_t steps = (K + 31) / 32, turns = (steps + U * KW - 1) / (U * KW);
    const int64_t s0 = turns * blockIdx.y / a.ksplit * (U * KW), end = turns * (blockIdx.y + 1) / a.ksplit * (U * KW);
    const int64_t s1 = (32 * tg < tv.count || TG == 1) ? (end < steps ? end : steps) : s0;
    const uint16_t *xrow[MT];
    int64_t place[MT];
    bool live[MT];
#pragma unroll
    for (int m = 0; m < MT; ++m) {
        if constexpr (TG == 1) {
            place[m] = tv.place;
            live[m] = tv.live;
            xrow[m] = a.X + tv.token * a.ldx;
        } else {
            const int tok = 32 * tg + 16 * m + r16;
            live[m] = tok < tv.count;
            place[m] = tv.first + (live[m] ? tok : tv.count - 1);
            xrow[m] = a.X + int64_t(a.plan[a.l.order + place[m]]) * a.ldx;
        }
    }
    // ranks past the adapter's own read its first (rows of a product do not mix)
    const uint16_t *arow[VB];
    int rin[VB];  // of the lane's four results, those within the adapter's rank
#pragma unroll
    for (int b = 0; b < VB; ++b) {
        const int v = v0 + b < a.nv ? v0 + b : a.nv - 1, pi = v / a.rb, r0 = 16 * (v - pi * a.rb);
        const Proj &p = a.p[pi];
        const int re = rank_of(p, tv.adapter, a.rank);
        rin[b] = re - r0 - 4 * g;
        arow[b] = p.A + adapter_row(tv.adapter, a.rank, r0 + r16, re) * K;
    }
    f32x4_t acc[MT][VB];
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int b = 0; b < VB; ++b) acc[m][b] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
    frag_t x[U][MT], w[U][VB];
    auto fetch = [&](int u, int64_t s) {
        const int64_t k = 32 * (s < s1 ? s : s0) + 8 * g;
#pragma unroll
        for (int m = 0; m < MT; ++m) x[u][m] = raw8<EVEN>(xrow[m], k, K);
#pragma unroll
        for (int b = 0; b < VB; ++b) w[u][b] = raw8<EVEN>(arow[b], k, K);
    };
    // `last`: the wave's last turn, the only one that may reach past d_in or the
    // block's steps. Both operands are masked there: what stands for the missing
    // ones are values of the row, and 0 times an infinity is no 0.
    auto product = [&](int u, int64_t s, auto last) {
        constexpr bool LAST = decltype(last)::value;
        const int64_t left = (s < s1) ? K - 32 * s - 8 * g : 0;
        frag_t xm[MT], wm[VB];
#pragma unroll
        for (int m = 0; m < MT; ++m) xm[m] = LAST ? first8<EVEN>(x[u][m], left) : x[u][m];
#pragma unroll
        for (int b = 0; b < VB; ++b) wm[b] = LAST ? first8<EVEN>(w[u][b], left) : w[u][b];
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
            for (int b = 0; b < VB; ++b) acc[m][b] = mfma(wm[b], xm[m], acc[m][b]);
    };
    int64_t s = s0 + U * kw;
    if (s < s1) {
#pragma unroll
        for (int u = 0; u < U; ++u) fetch(u, s + u);
        for (; s + U * KW < s1; s += U * KW)
#pragma unroll
            for (int u = 0; u < U; ++u) {
                product(u, s + u, std::false_type{});
                fetch(u, s + U * KW + u);
            }
#pragma unroll
        for (int u = 0; u < U; ++u) product(u, s + u, std::true_type{});
    }
    // lane: ranks 4 g .. + 3 of a block, of token r16; the waves along d_in added in order
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int b = 0; b < VB; ++b) s_acc[wave][m * VB + b][lane] = acc[m][b];
    __syncthreads();
    float *part = a.part + int64_t(blockIdx.y) * a.nv * a.M * 16 + 4 * g;
#pragma unroll
    for (int q = 0; q < MT * VB; ++q) {
        const int m = q / VB, b = q - m * VB;
        if (q % KW != kw) continue;
        f32x4_t v = s_acc[KW * tg][q][lane];
#pragma unroll
        for (int k = 1; k < KW; ++k) v += s_acc[KW * tg + k][q][lane];
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = e < rin[b] ? v[e] : 0.0f;
        if (live[m] && v0 + b < a.nv) *reinterpret_cast<f32x4_t *>(part + (int64_t(v0 + b) * a.M + place[m]) * 16) = v;
    }
}

// Sum over `splits` partial sums, in order, of eight values of block v from
// rank r (0 or 8) on.
__device__ __forceinline__ void part_sum(const AdArgs &a, int splits, int v, int64_t place, int r, float (&out)[8])
{
    const float *q = a.part + (int64_t(v) * a.M + place) * 16 + r;
    const int64_t step = int64_t(a.nv) * a.M * 16;
    f32x4_t x = *reinterpret_cast<const f32x4_t *>(q), y = *reinterpret_cast<const f32x4_t *>(q + 4);
#pragma unroll 8
    for (int z = 1; z < splits; ++z) {
        x += *reinterpret_cast<const f32x4_t *>(q + z * step);
        y += *reinterpret_cast<const f32x4_t *>(q + z * step + 4);
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        out[e] = x[e];
        out[4 + e] = y[e];
    }
}

// ---------------------------------------------------------------------------
// 64 columns of 16 tokens, read and written: lane (g, r16) has 16 columns of its
// token in runs of RUN (16 bytes of the type in memory), run q from column 4 RUN
// q + RUN g on, so that a wave's 16-byte words are 64 bytes next to each other.
// Value e of the lane is the sum that a product of 16 x 16 leaves in register e %
// 4 of block e / 4 when row i of block j of W is column run_column(i, j).
// ---------------------------------------------------------------------------
template <int RUN>
__device__ __forceinline__ int run_column(int i, int j)  // row i of block j
{
    return RUN == 8 ? 32 * (j >> 1) + 8 * (i >> 2) + 4 * (j & 1) + (i & 3) : 16 * j + i;
}

template <bool F32>
struct Row16 {
    u32x4_t w[F32 ? 4 : 2];
};

// `p`: the lane's first column; `nc`: columns from there on that exist; `whole`:
// all of the wave's 64 do
template <bool F32, int RUN>
__device__ __forceinline__ Row16<F32> load_row(const void *p, int64_t nc, bool whole)
{
    static_assert(!F32 || RUN == 4, "words of four 32-bit values");
    Row16<F32> v;
#pragma unroll
    for (int q = 0; q < 16 / RUN; ++q) v.w[q] = zero_frag();
    if (whole) {
#pragma unroll
        for (int q = 0; q < 16 / RUN; ++q) v.w[q] = load16(static_cast<const char *>(p) + 64 * q);
        return v;
    }
#pragma unroll
    for (int q = 0; q < 16 / RUN; ++q) {
        const int64_t left = nc - 4 * RUN * q;
        const char *pq = static_cast<const char *>(p) + 64 * q;
        if (left >= RUN) {
            v.w[q] = load16(pq);
            continue;
        }
#pragma unroll
        for (int e = 0; e < RUN; ++e)
            if (e < left) {
                if constexpr (F32) v.w[q][e] = reinterpret_cast<const uint32_t *>(pq)[e];
                else v.w[q][e >> 1] |= uint32_t(reinterpret_cast<const uint16_t *>(pq)[e]) << (16 * (e & 1));
            }
    }
    return v;
}

template <bool F32>
__device__ __forceinline__ float row_value(const Row16<F32> &v, int e)
{
    if constexpr (F32) return __uint_as_float(v.w[e >> 2][e & 3]);
    const uint32_t w = v.w[e >> 3][(e >> 1) & 3];
    return __uint_as_float((e & 1) ? w & 0xffff0000u : w << 16);
}

template <bool F32, int RUN>
__device__ __forceinline__ void store_row(void *p, int64_t nc, const float (&v)[16])
{
    constexpr int ES = F32 ? 4 : 2;
#pragma unroll
    for (int q = 0; q < 16 / RUN; ++q) {
        const int64_t left = nc - 4 * RUN * q;
        char *pq = static_cast<char *>(p) + 4 * RUN * q * ES;
        const float *x = v + RUN * q;
        if (left >= RUN) {
            if constexpr (F32) {
#pragma unroll
                for (int k = 0; k < RUN / 4; ++k)
                    reinterpret_cast<any_f32x4_t *>(pq)[k] = f32x4_t{x[4 * k], x[4 * k + 1], x[4 * k + 2], x[4 * k + 3]};
            } else {
                *reinterpret_cast<any_u32x4_t *>(pq) =
                    u32x4_t{pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]), pack_bf16x2(x[4], x[5]), pack_bf16x2(x[6], x[7])};
            }
        } else {
#pragma unroll
            for (int e = 0; e < RUN; ++e)
                if (e < left) {
                    if constexpr (F32) reinterpret_cast<float *>(pq)[e] = x[e];
                    else reinterpret_cast<uint16_t *>(pq)[e] = f32_to_bf16(x[e]);
                }
        }
    }
}

// ---------------------------------------------------------------------------
// expand: y = y0 + s B t. A block: a tile and a.ecols columns; a wave: 16 tokens
// (64-token tiles) over all of them, or every fourth 64 columns of all 16. t is
// summed once; then per 64 columns the wave has y0 and B of the next ones in
// flight. Bound by reading y0 and writing y (8192 tokens of 6144 columns at rank
// 16: 55 us, 3.7 TB/s of both). Reading ahead past a block's last columns, to
// spare the condition, made it 4 us slower.
// ---------------------------------------------------------------------------
template <int RB, bool EVEN, int TG, bool F32, bool DIRECT>
__global__ __launch_bounds__(AT) void adapters_expand(const AdArgs a)
{
    constexpr int PF = (RB == 1 && !DIRECT) ? 2 : 1;  // 64-column groups in flight (DIRECT: 14 us for 64 tokens, with two 18)
    __shared__ int s_tok[4][16];
    TileView tv;
    if (!tile_view<DIRECT, TG>(a, true, s_tok, tv)) return;
    const int t = threadIdx.x, lane = t & 63, g = lane >> 4, r16 = lane & 15;
    const int wave = __builtin_amdgcn_readfirstlane(t >> 6);
    const Proj &p = a.p[blockIdx.z];
    const int64_t C = p.d_out;
    const int64_t cb = int64_t(blockIdx.y) * a.ecols;
    if (cb >= C || (TG != 1 && 16 * wave >= tv.count)) return;
    const int64_t c0 = cb + (TG == 1 ? 64 * wave : 0), cstep = (TG == 1) ? 256 : 64;
    const int64_t c1 = (cb + a.ecols < C) ? cb + a.ecols : C;
    const int ad = tv.adapter;
    const bool keep = DIRECT && p.t && blockIdx.y == 0 && wave == 0 && tv.live;
    // rows without an adapter stay as they are in place
    if (ad < 0 && p.base == p.y && !keep) return;
    const int re = ad >= 0 ? rank_of(p, ad, a.rank) : 0;
    constexpr int64_t ES = F32 ? 4 : 2;
    constexpr int RUN = F32 ? 4 : 8;
    const char *base = static_cast<const char *>(p.base) + tv.token * p.ldb * ES;
    char *out = static_cast<char *>(p.y) + tv.token * p.ldy * ES;
    const uint16_t *B = p.B + int64_t(ad < 0 ? 0 : ad) * C * a.rank;
    const int r0 = 8 * (g & 1);  // the lane's ranks of a block
    // B: rows past d_out are its last (rows of a product do not mix), ranks past the
    // adapter's own are masked before the product (all of them where there is no
    // adapter: 0 times an infinity would be no 0)
    const bool part_rank = p.ranks != nullptr || a.rank % 16 != 0 || ad < 0;
    auto load_b = [&](int64_t c, frag_t (&w)[RB][4]) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int64_t cc = c + run_column<RUN>(r16, j);
            const int64_t row = (cc < C ? cc : C - 1) * a.rank;
#pragma unroll
            for (int b = 0; b < RB; ++b) {
                const int r = 16 * b + r0 < a.rank ? 16 * b + r0 : 0;
                w[b][j] = flat8<EVEN>(B, row + r, C * a.rank);
            }
        }
    };
    auto load_y = [&](int64_t c) {
        const int64_t col = c + RUN * g;
        return load_row<F32, RUN>(base + col * ES, (p.base && tv.live) ? C - col : 0, p.base && c + 64 <= C);
    };
    frag_t w[PF][RB][4];
    Row16<F32> y0[PF];
    auto load = [&](int q, int64_t c) {  // (past the block's columns: its first again)
        const int64_t cc = c < c1 ? c : c0;
        y0[q] = load_y(cc);
        load_b(cc, w[q]);
    };
#pragma unroll
    for (int q = 0; q < PF; ++q) load(q, c0 + q * cstep);
    // t in parts: the first and the second share a product (lanes g < 2 the
    // first), the third, for 32-bit results, has its own
    frag_t tf[RB], tf3[F32 ? RB : 1];
#pragma unroll
    for (int b = 0; b < RB; ++b) {
        tf[b] = zero_frag();
        if (F32) tf3[b] = zero_frag();
        if constexpr (DIRECT) {
            float v[8] = {0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f};
            if (ad >= 0) part_sum(a, a.ksplit, int(blockIdx.z) * RB + b, tv.place, r0, v);
            if (keep && g < 2)
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    if (16 * b + r0 + e < a.rank) p.t[tv.token * a.rank + 16 * b + r0 + e] = v[e];
            const float sc = ad >= 0 ? scale_of(p, ad) : 0.0f;
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] *= sc;
            frag_t part[3];
            split3(v, part);
            tf[b] = (g < 2) ? part[0] : part[1];
            if (F32 && g < 2) tf3[b] = part[2];
        } else if (ad >= 0) {
            const uint16_t *q = a.hl + (int64_t(int(blockIdx.z) * RB + b) * a.M + tv.place) * 48 + r0;
            tf[b] = *reinterpret_cast<const frag_t *>(q + 16 * (g >> 1));
            if (F32 && g < 2) tf3[b] = *reinterpret_cast<const frag_t *>(q + 32);
        }
    }
    if (ad < 0 && p.base == p.y) return;
    for (int64_t cq = c0; cq < c1; cq += PF * cstep)
#pragma unroll
        for (int q = 0; q < PF; ++q) {
            const int64_t c = cq + q * cstep;
            if (c >= c1) break;
            f32x4_t acc[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) acc[j] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
            if (part_rank)
#pragma unroll
                for (int b = 0; b < RB; ++b) {
                    const frag_t m = first8<false>(frag_t{~0u, ~0u, ~0u, ~0u}, re - 16 * b - r0);
#pragma unroll
                    for (int j = 0; j < 4; ++j) w[q][b][j] &= m;
                }
#pragma unroll
            for (int b = 0; b < RB; ++b)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    if (F32) acc[j] = mfma(w[q][b][j], tf3[b], acc[j]);
                    acc[j] = mfma(w[q][b][j], tf[b], acc[j]);
                }
            float v[16];
#pragma unroll
            for (int e = 0; e < 16; ++e) v[e] = row_value<F32>(y0[q], e) + acc[e >> 2][e & 3];
            if (cq + PF * cstep < c1) load(q, c + PF * cstep);
            const int64_t col = c + RUN * g;
            if (tv.live) store_row<F32, RUN>(out + col * ES, C - col, v);
        }
}

// ---------------------------------------------------------------------------
// Transposed reads of LDS tiles of 16-bit values: eight rows (k) of the lane's
// column, two reads of four.
// ---------------------------------------------------------------------------
typedef short s16x4_t __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) s16x4_t lds_s16x4_t;

__device__ __forceinline__ frag_t read_tr(const uint8_t *p, int four)
{
    typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
    const u32x2 a = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_t *)p));
    const u32x2 b = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_t *)(p + four)));
    return frag_t{a[0], a[1], b[0], b[1]};
}

// ---------------------------------------------------------------------------
// dx: dx = dx0 + sum over the projections of A^T u. A block: a tile and 128
// columns, 16 tokens a wave (16-token tiles: 256, 64 a wave). Per rank block 16
// rows of A are staged in LDS (two blocks of eight ranks, [pair of 16-column
// groups][rank][64 bytes], the groups swapped in ranks 8 to 15: the rows that
// half a wave reads together fall on all banks once) and read transposed. The
// columns are permuted on the way in (run_column). Bound by reading dx0 and
// writing dx (8192 tokens of 4096 columns, three projections of rank 16: 42 us, 3.2
// TB/s of both).
// ---------------------------------------------------------------------------
constexpr int DX_COLS = 128;

template <bool EVEN, int TG, bool F32>
__global__ __launch_bounds__(AT) void adapters_dx(const AdArgs a)
{
    constexpr int BC = (TG == 1) ? 256 : DX_COLS, NC = (TG == 1) ? 1 : BC / 64;  // columns of a block, 64-column groups of a wave
    constexpr int HALF = 16 * BC, SQ = BC / 128;                                 // bytes of eight ranks, 16-byte words a thread
    __shared__ __attribute__((aligned(16))) uint8_t s_a[2][2 * HALF];
    TileView tv;
    if (!tile_view<false, TG>(a, true, nullptr, tv)) return;
    const int t = threadIdx.x, lane = t & 63, g = lane >> 4, r16 = lane & 15;
    const int wave = __builtin_amdgcn_readfirstlane(t >> 6);
    const int64_t C = a.d_in, cb = int64_t(blockIdx.y) * BC;
    const int ad = tv.adapter;
    if (ad < 0 && a.dx0 == a.dx) return;
    const int64_t c0 = cb + (TG == 1 ? 64 * wave : 0);
    // (a wave without tokens helps to stage)
    const bool idle = TG != 1 && 16 * wave >= tv.count;
    Row16<false> x0[NC];
#pragma unroll
    for (int c = 0; c < NC; ++c) {
        const int64_t col = c0 + 64 * c + 8 * g;
        x0[c] = load_row<false, 8>(a.dx0 + tv.token * a.lddx0 + col, (a.dx0 && tv.live) ? C - col : 0,
                                        a.dx0 && c0 + 64 * c + 64 <= C);
    }
    f32x4_t acc[NC][4];
#pragma unroll
    for (int c = 0; c < NC; ++c)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[c][j] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
    if (ad >= 0) {
        frag_t st[SQ];
        int re = 0;  // ranks of the block in flight
        auto fetch = [&](int v) {
            const int pi = v / a.rb, b = v - pi * a.rb;
            const Proj &p = a.p[pi];
            const int own = rank_of(p, ad, a.rank);
            re = own - 16 * b;
#pragma unroll
            for (int q = 0; q < SQ; ++q) {
                const int w = t + AT * q, r = w / (BC / 8);
                st[q] = raw8<EVEN>(p.A + adapter_row(ad, a.rank, 16 * b + r, own) * C, cb + 8 * (w % (BC / 8)), C);
            }
        };
        fetch(0);
        const int key = 4 * (g & 1) + (r16 >> 2);
        const int t0 = key * 64 + 8 * (r16 & 3) + 32 * (g & 1), t1 = t0 ^ 32;
        for (int v = 0; v < a.nv; ++v) {
            uint8_t *sa = s_a[v & 1];
#pragma unroll
            for (int q = 0; q < SQ; ++q) {
                // rank k, columns 8 cc ..: rows 4 i .. of blocks f and f + 1 (run_column)
                const int w = t + AT * q, k = w / (BC / 8), cc = w % (BC / 8), kk = 4 * (k >> 3) + (k & 3);
                const int i = cc & 3, f = 4 * (cc >> 3) + 2 * ((cc >> 2) & 1);
                uint8_t *d = sa + ((k >> 2) & 1) * HALF + (f >> 1) * 512 + kk * 64 + 8 * i;
                const int swap = 32 * (kk >> 2);
                const frag_t x = first8<true>(st[q], k < re);  // (columns past d_in are not written)
                *reinterpret_cast<uint2 *>(d + swap) = make_uint2(x[0], x[1]);
                *reinterpret_cast<uint2 *>(d + (32 - swap)) = make_uint2(x[2], x[3]);
            }
            __syncthreads();  // (the buffer of v is written again at v + 2, past v + 1's barrier)
            if (v + 1 < a.nv) fetch(v + 1);
            if (idle) continue;
            const uint16_t *q = a.hl + (int64_t(v) * a.M + tv.place) * 48 + 8 * (g & 1);
            const frag_t uf = *reinterpret_cast<const frag_t *>(q + 16 * (g >> 1));
            const frag_t u3 = (F32 && g < 2) ? *reinterpret_cast<const frag_t *>(q + 32) : zero_frag();
#pragma unroll
            for (int c = 0; c < NC; ++c)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int f = 4 * c + j;
                    const frag_t w = read_tr(sa + (TG == 1 ? wave * 1024 : 0) + ((f & 1) ? t1 : t0) + (f >> 1) * 512, HALF);
                    if (F32) acc[c][j] = mfma(w, u3, acc[c][j]);
                    acc[c][j] = mfma(w, uf, acc[c][j]);
                }
        }
    }
    if (!tv.live) return;
#pragma unroll
    for (int c = 0; c < NC; ++c) {
        const int64_t col = c0 + 64 * c + 8 * g;
        float v[16];
#pragma unroll
        for (int e = 0; e < 16; ++e) v[e] = row_value<false>(x0[c], e) + acc[c][e >> 2][e & 3];
        store_row<F32, 8>(static_cast<char *>(a.dx) + (tv.token * a.lddx + col) * (F32 ? 4 : 2), C - col, v);
    }
}

// ---------------------------------------------------------------------------
// dy pass: of a piece's tokens, dB[c][r] = sum_m dy[m][c] (s t)[m][r] and the
// partial u[m][r] = sum over the block's 256 columns of dy[m][c] B[c][r], from
// one reading of dy. Per step of 64 tokens the block stages 64 x 256 of dy and s
// t in three parts in LDS, and holds the next two steps' in registers. For dB (a
// wave: 64 columns, all tokens) both are read transposed, tokens along the depth;
// for u (a wave: 16 tokens, all columns) dy is read as it lies and the block's
// 256 x rank of B, staged once, transposed. 64 tokens a step keep 32 KiB of dy
// in flight per block (8192 tokens of 6144 columns at rank 16: 32 us, 3.1 TB/s of
// dy); with 32 the loads' latency showed (83 us for 8192 tokens of q, k and v).
//
// LDS rows of dy: a wave's 64 columns, 128 bytes, in 32-byte groups; group q of
// row k lies at q ^ key(k), so that the eight rows that half a wave reads
// together fall on different banks. The others: 32-byte rows of 16 values.
// ---------------------------------------------------------------------------
constexpr int OUT_COLS = 256, OUT_STEP = 64, OUT_AHEAD = 2;  // columns and tokens of a step, steps in flight

__device__ __forceinline__ int out_key(int k) { return ((k >> 1) & 1) | (((k >> 3) & 1) << 1); }

// The wave's 64 rows x 64 columns from k0 of the piece on: lane -> row lane / 8
// (+ 8 i), columns c + 8 (lane % 8) .. The rows' tokens are read a step before
// (out_tokens), so that no load waits for another.
__device__ __forceinline__ void out_tokens(const int32_t *order, int k0, int count, int32_t (&tok)[8])
{
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int k = k0 + 8 * i + (lane >> 3);
        tok[i] = order[k < count ? k : 0];
    }
}

template <bool EVEN>
__device__ __forceinline__ void out_fetch(const uint16_t *S, int64_t ld, const int32_t (&tok)[8], int64_t c, int64_t C,
                                          frag_t (&sv)[8])
{
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int i = 0; i < 8; ++i) sv[i] = raw8<EVEN>(S + int64_t(tok[i]) * ld, c + 8 * (lane & 7), C);
}

template <bool EVEN>
__device__ __forceinline__ void out_stage(uint8_t *ss, const frag_t (&sv)[8], int k0, int count, int64_t c, int64_t C)
{
    const int lane = threadIdx.x & 63;
    const int64_t left = C - c - 8 * (lane & 7);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int k = 8 * i + (lane >> 3);
        *reinterpret_cast<frag_t *>(ss + k * 128 + ((((lane & 7) >> 1) ^ out_key(k)) << 5) + ((lane & 1) << 4)) =
            first8<EVEN>(sv[i], k0 + k < count ? left : 0);
    }
}

// Where a piece's result goes: the gradient itself (an adapter's only piece), or
// its slot.
struct OutPlace {
    float *to;
    bool add;
};

__device__ __forceinline__ OutPlace out_place(const AdArgs &a, const int4 &piece, int pi, bool is_a)
{
    const Proj &p = a.p[pi];
    if (piece.w < 0) return {(is_a ? p.dA : p.dB) + int64_t(piece.x) * a.rank * (is_a ? a.d_in : p.d_out), a.accumulate != 0};
    float *o = a.slots + int64_t(piece.w) * a.slot_floats + (is_a ? int64_t(a.rank) * p.d_out : 0);
    for (int q = 0; q < pi; ++q) o += int64_t(a.rank) * (a.p[q].d_out + a.d_in);
    return {o, false};
}

template <int RB, bool EVEN>
__global__ __launch_bounds__(AT) void adapters_dy(const AdArgs a)
{
    constexpr int PF = (RB <= 2) ? OUT_AHEAD : 1;  // steps in flight
    __shared__ __attribute__((aligned(16))) uint8_t s_s[4][OUT_STEP * 128];
    __shared__ __attribute__((aligned(16))) uint8_t s_q[RB][3][OUT_STEP * 32];
    __shared__ __attribute__((aligned(16))) uint8_t s_b[RB][OUT_COLS * 32];
    if (int(blockIdx.x) >= a.plan[2]) return;
    const int4 piece = reinterpret_cast<const int4 *>(a.plan + a.l.pieces)[blockIdx.x];
    const int pi = blockIdx.z;
    const Proj &p = a.p[pi];
    const int64_t C = p.d_out, cb = int64_t(blockIdx.y) * OUT_COLS;
    if (cb >= C) return;
    const int t = threadIdx.x, lane = t & 63, g = lane >> 4, r16 = lane & 15;
    const int wave = __builtin_amdgcn_readfirstlane(t >> 6);
    const int64_t c0 = cb + 64 * wave;
    const uint16_t *S = static_cast<const uint16_t *>(p.base);
    const int32_t *order = a.plan + a.l.order + piece.y;
    const int re = rank_of(p, piece.x, a.rank);
    const float sc = scale_of(p, piece.x);
    // s t: eight ranks of a row a thread
    constexpr int QV = (OUT_STEP * 2 * RB + AT - 1) / AT;
    frag_t sv[PF][8];
    float qv[PF][QV][8];
    int32_t tok[2][8], qtok[2][QV];
    auto tokens = [&](int k0, int h) {
        out_tokens(order, k0, piece.z, tok[h]);
#pragma unroll
        for (int q = 0; q < QV; ++q) {
            const int k = k0 + (t + AT * q) / (2 * RB);
            qtok[h][q] = order[k < piece.z ? k : 0];
        }
    };
    // (loads return in order: the next step's tokens go ahead of this one's rows)
    auto fetch = [&](int k0, int i) {
        const int h = i & 1;
        tokens(k0 + OUT_STEP, 1 - h);
        out_fetch<EVEN>(S, p.ldb, tok[h], c0, C, sv[i % PF]);
#pragma unroll
        for (int q = 0; q < QV; ++q) {
            const int w = t + AT * q, row = w / (2 * RB), r = 8 * (w - row * 2 * RB);
            const float *tr = p.t + int64_t(qtok[h][q]) * a.rank;
            if constexpr (EVEN) {  // (rank a multiple of 8)
                const any_f32x4_t *t4 = reinterpret_cast<const any_f32x4_t *>(tr + (r < a.rank ? r : 0));
                const f32x4_t u = t4[0], v = t4[1];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    qv[i % PF][q][e] = u[e];
                    qv[i % PF][q][4 + e] = v[e];
                }
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e) qv[i % PF][q][e] = tr[r + e < a.rank ? r + e : 0];
            }
        }
    };
    tokens(0, 0);
#pragma unroll
    for (int i = 0; i < PF; ++i) fetch(i * OUT_STEP, i);
    // B: row (column of dy) t, 16 ranks of every block
    {
        const bool in = cb + t < C;
        const uint16_t *br = p.B + (int64_t(piece.x) * C + (in ? cb + t : 0)) * a.rank;
#pragma unroll
        for (int b = 0; b < RB; ++b)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int r = 16 * b + 8 * h;
                const frag_t v = first8<false>(flat8<EVEN>(br, r < a.rank ? r : 0, (C - (in ? cb + t : 0)) * a.rank), in ? re - r : 0);
                *reinterpret_cast<frag_t *>(s_b[b] + t * 32 + 16 * h) = v;
            }
    }
    f32x4_t acc[4][RB];
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int b = 0; b < RB; ++b) acc[i][b] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
    uint8_t *ss = s_s[wave];
    const int kr = 8 * g + (r16 >> 2), key = out_key(kr);  // the lane's row in a transposed read
    const int quad = (r16 & 3) << 3;
    auto step = [&](int k0, int cur) {
        __syncthreads();  // the last step's reads are over
        out_stage<EVEN>(ss, sv[cur % PF], k0, piece.z, c0, C);
#pragma unroll
        for (int q = 0; q < QV; ++q) {
            const int w = t + AT * q, row = w / (2 * RB), r = 8 * (w - row * 2 * RB);
            if (row >= OUT_STEP) continue;
            float x[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = (k0 + row < piece.z && r + e < re) ? sc * qv[cur % PF][q][e] : 0.0f;
            frag_t part[3];
            split3(x, part);
#pragma unroll
            for (int h = 0; h < 3; ++h) *reinterpret_cast<frag_t *>(s_q[r >> 4][h] + row * 32 + 2 * (r & 8)) = part[h];
        }
        __syncthreads();
        if (k0 + PF * OUT_STEP < piece.z) fetch(k0 + PF * OUT_STEP, cur + PF);
#pragma unroll
        for (int d = 0; d < 2; ++d) {  // 32 tokens
            if (k0 + 32 * d >= piece.z) break;
            frag_t sf[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) sf[i] = read_tr(ss + (32 * d + kr) * 128 + ((i ^ key) << 5) + quad, 4 * 128);
#pragma unroll
            for (int b = 0; b < RB; ++b)
#pragma unroll
                for (int h = 0; h < 3; ++h) {
                    const frag_t qf = read_tr(s_q[b][h] + (32 * d + kr) * 32 + quad, 4 * 32);
#pragma unroll
                    for (int i = 0; i < 4; ++i) acc[i][b] = mfma(sf[i], qf, acc[i][b]);
                }
        }
        // u of tokens 16 wave .. + 15 over the block's columns
        const int row = 16 * wave + r16;
        if (k0 + 16 * wave < piece.z) {
            f32x4_t u[RB];
#pragma unroll
            for (int b = 0; b < RB; ++b) u[b] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int h = 0; h < 8; ++h) {
                const frag_t rf = *reinterpret_cast<const frag_t *>(
                    s_s[h >> 1] + row * 128 + (((2 * (h & 1) + (g >> 1)) ^ out_key(row)) << 5) + ((g & 1) << 4));
#pragma unroll
                for (int b = 0; b < RB; ++b) u[b] = mfma(read_tr(s_b[b] + (32 * h + kr) * 32 + quad, 4 * 32), rf, u[b]);
            }
            if (k0 + row < piece.z)
#pragma unroll
                for (int b = 0; b < RB; ++b)
                    *reinterpret_cast<f32x4_t *>(
                        a.part + ((int64_t(blockIdx.y) * a.nv + pi * RB + b) * a.M + piece.y + k0 + row) * 16 + 4 * g) = u[b];
        }
    };
    for (int k0 = 0; k0 < piece.z; k0 += 2 * OUT_STEP) {
        step(k0, 0);
        if (k0 + OUT_STEP < piece.z) step(k0 + OUT_STEP, 1);
    }
    // lane: columns c0 + 16 i + 4 g .. + 3 at rank 16 b + r16; 0 past the adapter's
    // rank, also where dy is not finite (its sum there is of 0 times an infinity)
    const OutPlace o = out_place(a, piece, pi, false);
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int b = 0; b < RB; ++b) {
            const int r = 16 * b + r16;
            const int64_t c = c0 + 16 * i + 4 * g;
            if (r >= a.rank) continue;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                if (c + e >= C) break;
                float *q = o.to + (c + e) * a.rank + r;
                const float v = r < re ? acc[i][b][e] : 0.0f;
                *q = o.add ? *q + v : v;
            }
        }
}

// s times the partial sums of t (or u) in order, in three bf16 parts, zero past
// an adapter's rank; t itself is kept where it is asked for. One thread per eight
// ranks of a token; z: projection.
template <bool BACK>
__global__ __launch_bounds__(AT) void adapters_parts(const AdArgs a)
{
    const int groups = 2 * a.rb;
    const int64_t i = int64_t(blockIdx.x) * AT + threadIdx.x;
    const int64_t place = i / groups;
    const int r = int(i - place * groups) * 8;
    const int32_t *seg = a.plan + a.l.seg;
    if (place >= a.M) return;
    const int pi = blockIdx.z, v = pi * a.rb + (r >> 4);
    const Proj &p = a.p[pi];
    const bool none = place >= seg[a.n];
    float x[8] = {0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f};
    int lo = 0, hi = a.n;
    if (!none) {
        part_sum(a, BACK ? int((p.d_out + OUT_COLS - 1) / OUT_COLS) : a.ksplit, v, place, r & 8, x);
        // its adapter: the last whose first place is not past it
        while (hi - lo > 1) {
            const int mid = (lo + hi) / 2;
            if (seg[mid] <= place) lo = mid;
            else hi = mid;
        }
    }
    if (!BACK && p.t) {
        float *t = p.t + int64_t(a.plan[a.l.order + place]) * a.rank + r;
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (r + e < a.rank) t[e] = x[e];
    }
    if (none) return;
    const int re = rank_of(p, lo, a.rank);
    const float sc = scale_of(p, lo);
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = (r + e < re) ? sc * x[e] : 0.0f;
    frag_t part[3];
    split3(x, part);
    uint16_t *q = a.hl + (int64_t(v) * a.M + place) * 48 + (r & 8);
#pragma unroll
    for (int k = 0; k < 3; ++k) *reinterpret_cast<frag_t *>(q + 16 * k) = part[k];
}

// ---------------------------------------------------------------------------
// dA: of a piece's tokens, dA[r][c] = sum_m u[m][r] x[m][c], for VB rank blocks
// of the group from one reading of x; staged and read as dB's operands. Bound by
// the turn of a step, loads to LDS to products, with few waves beside each other
// (8192 tokens of 4096 columns, three blocks: 41 us, 1.7 TB/s of x; pieces of M / 24
// tokens for more blocks cost more in partial sums than they gain).
// ---------------------------------------------------------------------------
template <int VB, bool EVEN>
__global__ __launch_bounds__(AT) void adapters_da(const AdArgs a)
{
    constexpr int PF = OUT_AHEAD;  // steps in flight
    __shared__ __attribute__((aligned(16))) uint8_t s_s[4][OUT_STEP * 128];
    __shared__ __attribute__((aligned(16))) uint8_t s_q[VB][3][OUT_STEP * 32];
    if (int(blockIdx.x) >= a.plan[2]) return;
    const int4 piece = reinterpret_cast<const int4 *>(a.plan + a.l.pieces)[blockIdx.x];
    const int64_t C = a.d_in, cb = int64_t(blockIdx.y) * OUT_COLS;
    const int t = threadIdx.x, lane = t & 63, g = lane >> 4, r16 = lane & 15;
    const int wave = __builtin_amdgcn_readfirstlane(t >> 6);
    const int64_t c0 = cb + 64 * wave;
    const int v0 = int(blockIdx.z) * VB;
    const int32_t *order = a.plan + a.l.order + piece.y;
    f32x4_t acc[4][VB];
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int b = 0; b < VB; ++b) acc[i][b] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
    uint8_t *ss = s_s[wave];
    constexpr int QR = OUT_STEP * 6, QV = (VB * QR + AT - 1) / AT;  // 16-byte words of u's parts, of a block
    frag_t sv[PF][8], qv[PF][QV];
    int32_t tok[2][8];
    out_tokens(order, 0, piece.z, tok[0]);
    auto fetch = [&](int k0, int i) {
        out_tokens(order, k0 + OUT_STEP, piece.z, tok[1 - (i & 1)]);
        out_fetch<EVEN>(a.X, a.ldx, tok[i & 1], c0, C, sv[i % PF]);
#pragma unroll
        for (int q = 0; q < QV; ++q) {
            const int w = t + AT * q, b = w / QR, x = w - QR * b;
            const int v = v0 + b < a.nv ? v0 + b : v0;
            qv[i % PF][q] = reinterpret_cast<const frag_t *>(a.hl + (int64_t(v) * a.M + piece.y) * 48)[k0 + x / 6 < piece.z ? 6 * k0 + x : 0];
        }
    };
#pragma unroll
    for (int i = 0; i < PF; ++i) fetch(i * OUT_STEP, i);
    const int kr = 8 * g + (r16 >> 2), key = out_key(kr), quad = (r16 & 3) << 3;
    auto step = [&](int k0, int cur) {
        __syncthreads();  // the last step's reads are over
        out_stage<EVEN>(ss, sv[cur % PF], k0, piece.z, c0, C);
#pragma unroll
        for (int q = 0; q < QV; ++q) {
            // parts of a row: 0 0 1 1 2 2
            const int w = t + AT * q, b = w / QR, x = w - QR * b, row = x / 6, c = x - 6 * row;
            if (b < VB) *reinterpret_cast<frag_t *>(s_q[b][c >> 1] + row * 32 + 16 * (c & 1)) = first8<true>(qv[cur % PF][q], k0 + row < piece.z);
        }
        __syncthreads();
        if (k0 + PF * OUT_STEP < piece.z) fetch(k0 + PF * OUT_STEP, cur + PF);
#pragma unroll
        for (int d = 0; d < 2; ++d) {  // 32 tokens
            if (k0 + 32 * d >= piece.z) break;
            frag_t sf[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) sf[i] = read_tr(ss + (32 * d + kr) * 128 + ((i ^ key) << 5) + quad, 4 * 128);
#pragma unroll
            for (int b = 0; b < VB; ++b)
#pragma unroll
                for (int h = 0; h < 3; ++h) {
                    const frag_t qf = read_tr(s_q[b][h] + (32 * d + kr) * 32 + quad, 4 * 32);
#pragma unroll
                    for (int i = 0; i < 4; ++i) acc[i][b] = mfma(sf[i], qf, acc[i][b]);
                }
        }
    };
    for (int k0 = 0; k0 < piece.z; k0 += 2 * OUT_STEP) {
        step(k0, 0);
        if (k0 + OUT_STEP < piece.z) step(k0 + OUT_STEP, 1);
    }
#pragma unroll
    for (int b = 0; b < VB; ++b) {
        const int v = v0 + b;
        if (v >= a.nv) break;
        const int pi = v / a.rb, r = 16 * (v - pi * a.rb) + r16;
        if (r >= a.rank) continue;
        const bool in = r < rank_of(a.p[pi], piece.x, a.rank);  // (as dB: 0 past the adapter's rank)
        const OutPlace o = out_place(a, piece, pi, true);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int64_t c = c0 + 16 * i + 4 * g;
            float *q = o.to + int64_t(r) * C + c;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float v = in ? acc[i][b][e] : 0.0f;
                if (c + e < C) q[e] = o.add ? q[e] + v : v;
            }
        }
    }
}

// Adapters of several pieces: their sum in order; of none: zero. One block per
// 1024 values; y: adapter; z: 2 projection + (1 for dA).
__global__ __launch_bounds__(AT) void adapters_pieces(const AdArgs a)
{
    const int ad = blockIdx.y, pi = int(blockIdx.z) >> 1, is_a = int(blockIdx.z) & 1;
    const Proj &p = a.p[pi];
    const int32_t *pf = a.plan + a.l.seg + a.n + 2;
    const int n0 = pf[ad], n1 = pf[ad + 1];
    if (n1 - n0 == 1 || (n1 == n0 && a.accumulate)) return;
    const int64_t total = int64_t(a.rank) * (is_a ? a.d_in : p.d_out);
    const int64_t i0 = int64_t(blockIdx.x) * 4 * AT;
    if (i0 >= total) return;
    float *out = (is_a ? p.dA : p.dB) + ad * total;
    int64_t off = is_a ? int64_t(a.rank) * p.d_out : 0;
    for (int q = 0; q < pi; ++q) off += int64_t(a.rank) * (a.p[q].d_out + a.d_in);
    // the adapter's slots follow each other
    const float *src = nullptr;
    if (n1 > n0) src = a.slots + int64_t(reinterpret_cast<const int4 *>(a.plan + a.l.pieces)[n0].w) * a.slot_floats + off;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const int64_t i = i0 + e * AT + threadIdx.x;
        if (i >= total) break;
        float v = 0.0f;
        for (int q = 0; q < n1 - n0; ++q) v += src[q * a.slot_floats + i];
        out[i] = a.accumulate ? out[i] + v : v;
    }
}

// ---------------------------------------------------------------------------
// Host side.
// ---------------------------------------------------------------------------
struct AdLayout {
    int ksplit;
    size_t part, hl, slots, plan, total;
    int64_t slot_floats;
};

// Rank blocks that a launch over x takes at once, of nv: threes or fours. Two,
// three and four at once are within 9% of each other in the forward calls of 2000
// tokens of 4096 inputs (six blocks 39, 42, 40 us; twelve 76, 70, 70). In dA fewer are
// faster: the gradients of eight blocks take 90, 86 and 100 us, of six 73, 79 and 85.
int blocks_at_once(int nv) { return nv <= 4 ? nv : (nv % 3 == 0 ? 3 : 4); }

// Splits of d_in: until the launch has about 1024 blocks, each wave with a turn
// of 128 inputs (64-token tiles: two) or more.
int shrink_splits(int64_t tiles, int groups, int64_t K)
{
    return int(std::clamp<int64_t>(1024 / std::max<int64_t>(1, tiles * groups), 1, std::clamp<int64_t>(K / 512, 1, 16)));
}

AdLayout ad_layout(bool back, int64_t M, int64_t n, int np, int rank, int64_t d_in, const int64_t *d_out)
{
    const PlanLayout pl = plan_layout(M, n);
    AdLayout l{};
    const int nv = np * rank_blocks(rank), at_once = blocks_at_once(nv);
    int64_t widest = 0;
    for (int i = 0; i < np; ++i) {
        widest = std::max(widest, d_out[i]);
        l.slot_floats += int64_t(rank) * (d_in + d_out[i]);
    }
    l.slot_floats = (l.slot_floats + 3) / 4 * 4;
    l.ksplit = shrink_splits(M / pl.tile + 1, (nv + at_once - 1) / at_once, d_in);
    const int64_t parts = back ? (widest + OUT_COLS - 1) / OUT_COLS : l.ksplit;
    size_t at = 0;
    auto take = [&](size_t bytes) {
        const size_t p = at;
        at += align256(bytes);
        return p;
    };
    l.part = take(size_t(parts) * nv * size_t(M) * 16 * 4);
    if (back || M > DIRECT_TOKENS) l.hl = take(size_t(nv) * size_t(M) * 48 * 2);
    if (back) {
        l.slots = take(size_t(pl.max_slots) * size_t(l.slot_floats) * 4);
        if (M <= DIRECT_TOKENS) l.plan = take(size_t(pl.words) * 4);
    }
    l.total = at;
    return l;
}

template <bool EVEN>
hipError_t launch_shrink(const AdArgs &a, dim3 grid, int vb, bool direct, hipStream_t st)
{
#define BSQ_VB(N)                                                                                                        \
    case N:                                                                                                              \
        if (direct) hipLaunchKernelGGL((adapters_shrink<N, EVEN, 1, true>), grid, dim3(AT), 0, st, a);                    \
        else if (a.l.tile == 16) hipLaunchKernelGGL((adapters_shrink<N, EVEN, 1, false>), grid, dim3(AT), 0, st, a);      \
        else hipLaunchKernelGGL((adapters_shrink<N, EVEN, 4, false>), grid, dim3(AT), 0, st, a);                          \
        break;
    switch (vb) {
        BSQ_VB(1)
        BSQ_VB(2)
        BSQ_VB(3)
        BSQ_VB(4)
    }
#undef BSQ_VB
    return hipGetLastError();
}

template <bool EVEN, bool F32>
hipError_t launch_expand(const AdArgs &a, dim3 grid, bool direct, hipStream_t st)
{
#define BSQ_RB(N)                                                                                                        \
    case N:                                                                                                              \
        if (direct) hipLaunchKernelGGL((adapters_expand<N, EVEN, 1, F32, true>), grid, dim3(AT), 0, st, a);               \
        else if (a.l.tile == 16) hipLaunchKernelGGL((adapters_expand<N, EVEN, 1, F32, false>), grid, dim3(AT), 0, st, a); \
        else hipLaunchKernelGGL((adapters_expand<N, EVEN, 4, F32, false>), grid, dim3(AT), 0, st, a);                     \
        break;
    switch (a.rb) {
        BSQ_RB(1)
        BSQ_RB(2)
        BSQ_RB(4)
        BSQ_RB(8)
    }
#undef BSQ_RB
    return hipGetLastError();
}

template <bool EVEN>
hipError_t launch_dy(const AdArgs &a, dim3 grid, hipStream_t st)
{
    switch (a.rb) {
    case 1: hipLaunchKernelGGL((adapters_dy<1, EVEN>), grid, dim3(AT), 0, st, a); break;
    case 2: hipLaunchKernelGGL((adapters_dy<2, EVEN>), grid, dim3(AT), 0, st, a); break;
    case 4: hipLaunchKernelGGL((adapters_dy<4, EVEN>), grid, dim3(AT), 0, st, a); break;
    default: hipLaunchKernelGGL((adapters_dy<8, EVEN>), grid, dim3(AT), 0, st, a); break;
    }
    return hipGetLastError();
}

template <bool EVEN>
hipError_t launch_da(const AdArgs &a, int vb, dim3 grid, hipStream_t st)
{
    switch (vb) {
    case 1: hipLaunchKernelGGL((adapters_da<1, EVEN>), grid, dim3(AT), 0, st, a); break;
    case 2: hipLaunchKernelGGL((adapters_da<2, EVEN>), grid, dim3(AT), 0, st, a); break;
    case 3: hipLaunchKernelGGL((adapters_da<3, EVEN>), grid, dim3(AT), 0, st, a); break;
    default: hipLaunchKernelGGL((adapters_da<4, EVEN>), grid, dim3(AT), 0, st, a); break;
    }
    return hipGetLastError();
}

template <bool EVEN, bool F32>
hipError_t launch_dx(const AdArgs &a, dim3 grid, hipStream_t st)
{
    if (a.l.tile == 16) hipLaunchKernelGGL((adapters_dx<EVEN, 1, F32>), grid, dim3(AT), 0, st, a);
    else hipLaunchKernelGGL((adapters_dx<EVEN, 4, F32>), grid, dim3(AT), 0, st, a);
    return hipGetLastError();
}

unsigned blocks(int64_t n, int64_t per) { return unsigned((n + per - 1) / per); }

hipError_t run_plan(const int32_t *ids, int64_t M, int64_t n, void *buf, int32_t *err, hipStream_t st)
{
    PlanArgs a{};
    a.ids = ids;
    a.buf = static_cast<int32_t *>(buf);
    a.err = err;
    a.M = M;
    a.n = int(n);
    for (a.bits = 1; (int64_t(1) << a.bits) <= n; ++a.bits) {}
    a.l = plan_layout(M, n);
    const size_t lds = size_t(PLAN_WAVES) * size_t(n + 1) * 4;
    if (lds > 28 * 1024) {  // with the kernel's own 32 KiB past the default limit
        const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void *>(&adapters_plan_kernel),
                                                 hipFuncAttributeMaxDynamicSharedMemorySize, int(lds));
        if (e != hipSuccess) return e;
    }
    hipLaunchKernelGGL(adapters_plan_kernel, dim3(1), dim3(64 * PLAN_WAVES), lds, st, a);
    return hipGetLastError();
}

hipError_t run_forward(const AdaptersCall &c, AdArgs &a, int64_t widest, hipStream_t st)
{
    const bool direct = a.M <= DIRECT_TOKENS, f32 = c.y_dtype == BSQ_F32;
    for (int i = 0; i < c.np; ++i) {
        Proj &p = a.p[i];
        p.base = c.y0 ? c.y0[i] : nullptr;
        p.ldb = c.y0 ? c.ldy0[i] : 0;
        p.y = c.y[i];
        p.ldy = c.ldy[i];
    }
    const bool even_in = c.d_in % 8 == 0, even_rank = c.rank % 8 == 0;
    const unsigned tiles = unsigned(direct ? a.M : a.l.max_tiles);
    const int vb = blocks_at_once(a.nv);
    const dim3 sgrid(tiles, unsigned(a.ksplit), blocks(a.nv, vb));
    hipError_t e = even_in ? launch_shrink<true>(a, sgrid, vb, direct, st) : launch_shrink<false>(a, sgrid, vb, direct, st);
    if (e != hipSuccess) return e;
    if (!direct) {
        hipLaunchKernelGGL((adapters_parts<false>), dim3(blocks(a.M * 2 * a.rb, AT), 1, unsigned(c.np)), dim3(AT), 0, st, a);
        if ((e = hipGetLastError()) != hipSuccess) return e;
    }
    // columns of a block: t and the tile are read once for all of them, but few
    // tiles need many blocks to fill the compute units (64 tokens of 24576 columns: 2048
    // columns 14 us, 1024 17, 512 23)
    a.ecols = (a.l.tile == 16) ? 2048 : 256;
    while (a.ecols > 256 && int64_t(tiles) * c.np * blocks(widest, a.ecols) < 768) a.ecols /= 2;
    const dim3 egrid(tiles, blocks(widest, a.ecols), unsigned(c.np));
    if (f32) return even_rank ? launch_expand<true, true>(a, egrid, direct, st) : launch_expand<false, true>(a, egrid, direct, st);
    return even_rank ? launch_expand<true, false>(a, egrid, direct, st) : launch_expand<false, false>(a, egrid, direct, st);
}

hipError_t run_backward(const AdaptersCall &c, AdArgs &a, int64_t widest, hipStream_t st)
{
    // rows of dy, t and B in whole words of eight; rows of x and A
    bool even_dy = c.rank % 8 == 0;
    const bool even_in = c.d_in % 8 == 0;
    for (int i = 0; i < c.np; ++i) {
        Proj &p = a.p[i];
        p.base = c.dy[i];
        p.ldb = c.lddy[i];
        p.dA = c.dA[i];
        p.dB = c.dB[i];
        even_dy = even_dy && p.d_out % 8 == 0;
    }
    const dim3 dgrid(unsigned(a.l.max_pieces), blocks(widest, OUT_COLS), unsigned(c.np));
    hipError_t e = even_dy ? launch_dy<true>(a, dgrid, st) : launch_dy<false>(a, dgrid, st);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((adapters_parts<true>), dim3(blocks(a.M * 2 * a.rb, AT), 1, unsigned(c.np)), dim3(AT), 0, st, a);
    if ((e = hipGetLastError()) != hipSuccess) return e;
    const int vb = blocks_at_once(a.nv);
    const dim3 agrid(unsigned(a.l.max_pieces), blocks(c.d_in, OUT_COLS), blocks(a.nv, vb));
    if ((e = even_in ? launch_da<true>(a, vb, agrid, st) : launch_da<false>(a, vb, agrid, st)) != hipSuccess) return e;
    hipLaunchKernelGGL(adapters_pieces, dim3(blocks(int64_t(c.rank) * std::max(widest, c.d_in), 4 * AT), unsigned(a.n), unsigned(2 * c.np)),
                       dim3(AT), 0, st, a);
    if ((e = hipGetLastError()) != hipSuccess || !c.dx) return e;
    a.dx0 = static_cast<const uint16_t *>(c.dx0);
    a.dx = c.dx;
    a.lddx0 = c.lddx0;
    a.lddx = c.lddx;
    const bool f32 = c.dx_dtype == BSQ_F32;
    const dim3 xgrid(unsigned(a.l.max_tiles), blocks(c.d_in, a.l.tile == 16 ? 256 : DX_COLS), 1);
    if (f32) return even_in ? launch_dx<true, true>(a, xgrid, st) : launch_dx<false, true>(a, xgrid, st);
    return even_in ? launch_dx<true, false>(a, xgrid, st) : launch_dx<false, false>(a, xgrid, st);
}

// Reports ids that are no adapter's (up to DIRECT_TOKENS tokens have no plan).
__global__ __launch_bounds__(DIRECT_TOKENS) void adapters_check_kernel(const int32_t *ids, int64_t M, int n, int32_t *err)
{
    const int64_t m = threadIdx.x;
    if (m < M && ids[m] >= n) atomicOr(err, BSQ_DEVERR_BAD_SET);
}

}  // namespace

size_t adapters_plan_bytes(int64_t M, int64_t n) { return M <= DIRECT_TOKENS ? 0 : size_t(plan_layout(M, n).words) * 4; }

hipError_t launch_adapters_plan(const int32_t *ids, int64_t M, int64_t n, void *buf, int32_t *err, hipStream_t st)
{
    if (M > DIRECT_TOKENS) return run_plan(ids, M, n, buf, err, st);
    if (!err) return hipSuccess;
    hipLaunchKernelGGL(adapters_check_kernel, dim3(1), dim3(DIRECT_TOKENS), 0, st, ids, M, int(n), err);
    return hipGetLastError();
}

size_t adapters_ws_bytes(bool back, int64_t M, int64_t n, int np, int rank, int64_t d_in, const int64_t *d_out)
{
    return ad_layout(back, M, n, np, rank, d_in, d_out).total;
}

hipError_t launch_adapters(const AdaptersCall &c, hipStream_t st)
{
    const bool back = c.dy != nullptr;
    AdArgs a{};
    a.plan = static_cast<const int32_t *>(c.plan->buf);
    a.ids = c.plan->ids;
    a.M = c.plan->M;
    a.n = c.plan->n;
    a.l = plan_layout(a.M, a.n);
    int64_t d_out[BSQ_MAX_GROUP], widest = 0;
    for (int i = 0; i < c.np; ++i) widest = std::max(widest, d_out[i] = c.pools[i].d_out);
    const AdLayout l = ad_layout(back, a.M, a.n, c.np, c.rank, c.d_in, d_out);
    char *ws = static_cast<char *>(c.ws);
    a.X = static_cast<const uint16_t *>(c.X);
    a.ldx = c.ldx;
    a.d_in = c.d_in;
    a.np = c.np;
    a.rank = c.rank;
    a.rb = rank_blocks(c.rank);
    a.nv = a.np * a.rb;
    a.ksplit = l.ksplit;
    a.part = reinterpret_cast<float *>(ws + l.part);
    a.hl = reinterpret_cast<uint16_t *>(ws + l.hl);
    a.slots = reinterpret_cast<float *>(ws + l.slots);
    a.slot_floats = l.slot_floats;
    a.accumulate = c.accumulate;
    for (int i = 0; i < c.np; ++i) {
        const bsq_adapter_pool &q = c.pools[i];
        Proj &p = a.p[i];
        p.A = q.A;
        p.B = q.B;
        p.scale = q.scale;
        p.ranks = q.ranks;
        p.d_out = q.d_out;
        p.t = c.t ? c.t[i] : nullptr;
    }
    if (!back) return run_forward(c, a, widest, st);
    if (a.M <= DIRECT_TOKENS) {
        const hipError_t e = run_plan(a.ids, a.M, a.n, ws + l.plan, nullptr, st);
        if (e != hipSuccess) return e;
        a.plan = reinterpret_cast<const int32_t *>(ws + l.plan);
    }
    return run_backward(c, a, widest, st);
}

}  // namespace bsq
