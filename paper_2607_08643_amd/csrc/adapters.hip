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
//   shrink   a tile's t (or u): the long dimension is split over blocks and
//            waves, whose fp32 partial sums go to the workspace;
//   expand   sums those in order and adds s B t to a tile's rows of y (A^T u
//            to those of dx);
//   outer    dA and dB of a run of one adapter's tokens (a "piece"), whose
//            partial results are added in order where there are several.
//
// t and u are held in fp32 and enter the next product as bf16 parts: the value
// rounded, then what remains, rounded. For bf16 results two parts (2^-16 of the
// value is lost, and a rank block of 16 with its two parts fills one 32-deep
// product), for fp32 results three (2^-24).
#include <algorithm>

#include "gemm_common.h"

namespace bsq {
namespace {

constexpr int AT = 256;  // threads of a block: 4 waves
constexpr int PLAN_WAVES = 16;

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
    l.tile = adapters_tile(M);
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

// Inclusive scans over the block's threads of four counts.
__device__ __forceinline__ void block_scan4(int (&v)[4], int (*s_wave)[4])
{
    const int t = threadIdx.x, lane = t & 63, w = t >> 6;
#pragma unroll
    for (int q = 0; q < 4; ++q)
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const int o = __shfl_up(v[q], d);
            if (lane >= d) v[q] += o;
        }
    if (lane == 63)
#pragma unroll
        for (int q = 0; q < 4; ++q) s_wave[w][q] = v[q];
    __syncthreads();
    for (int k = 0; k < w; ++k)
#pragma unroll
        for (int q = 0; q < 4; ++q) v[q] += s_wave[k][q];
}

// A stable counting sort in one block: each wave counts a run of tokens into
// its own row of counters (lanes of equal keys are found by ballots over the
// key's bits; their first adds for all), the rows are scanned, and each wave
// goes over its run again to place its tokens. No atomics: the order, and with
// it every sum over tokens, is fixed.
__global__ __launch_bounds__(64 * PLAN_WAVES) void adapters_plan_kernel(const PlanArgs a)
{
    extern __shared__ int32_t s_cnt[];  // [PLAN_WAVES][n + 1]
    __shared__ int s_wave[PLAN_WAVES][4];
    const int t = threadIdx.x, lane = t & 63, w = t >> 6, nk = a.n + 1;
    int32_t *row = s_cnt + w * nk;
    for (int k = t; k < PLAN_WAVES * nk; k += 64 * PLAN_WAVES) s_cnt[k] = 0;
    __syncthreads();
    const int64_t per = ((a.M + PLAN_WAVES - 1) / PLAN_WAVES + 63) / 64 * 64;
    const int64_t lo = w * per, hi = (lo + per < a.M) ? lo + per : a.M;
    int32_t *order = a.buf + a.l.order;
    bool bad = false;
    // pass 0 counts, pass 1 places
    for (int pass = 0; pass < 2; ++pass) {
        for (int64_t m0 = lo; m0 < hi; m0 += 64) {
            const int64_t m = m0 + lane;
            const bool in = m < hi;
            const int32_t id = in ? a.ids[m] : -1;
            bad |= id >= a.n;
            const int key = (id >= 0 && id < a.n) ? id : a.n;
            uint64_t same = __ballot(in);
            for (int b = 0; b < a.bits; ++b) {
                const uint64_t ones = __ballot((key >> b) & 1);
                same &= ((key >> b) & 1) ? ones : ~ones;
            }
            const int before = __popcll(same & ((uint64_t(1) << lane) - 1));
            const bool first = in && before == 0;
            if (pass == 1 && in) order[row[key] + before] = int32_t(m);
            // (a wave's LDS operations run in order, so the reads above come first)
            if (first) row[key] += __popcll(same);
        }
        __syncthreads();
        if (pass == 1) break;
        // thread k: the counts of adapter k
        int total = 0;
        if (t < a.n)
            for (int v = 0; v < PLAN_WAVES; ++v) total += s_cnt[v * nk + t];
        const int T = int(a.l.tile), P = int(a.l.piece);
        const int nt = (total + T - 1) / T, np = (total + P - 1) / P, ns = (np > 1) ? np : 0;
        int v[4] = {total, nt, np, ns};
        block_scan4(v, s_wave);
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
            int4 *tl = reinterpret_cast<int4 *>(a.buf + a.l.tiles) + (v[1] - nt);
            for (int q = 0; q < nt; ++q) tl[q] = make_int4(t, start + q * T, total - q * T < T ? total - q * T : T, 0);
            int4 *pc = reinterpret_cast<int4 *>(a.buf + a.l.pieces) + (v[2] - np);
            for (int q = 0; q < np; ++q)
                pc[q] = make_int4(t, start + q * P, total - q * P < P ? total - q * P : P, ns ? v[3] - ns + q : -1);
        }
        // the last thread holds the sums: the tokens without an adapter follow
        __shared__ int s_all[4];
        if (t == 64 * PLAN_WAVES - 1)
            for (int q = 0; q < 4; ++q) s_all[q] = v[q];
        __syncthreads();
        const int live = s_all[0], none = int(a.M) - live, nnt = (none + T - 1) / T;
        if (t == 0) {
            int at = live;
            for (int q = 0; q < PLAN_WAVES; ++q) {
                const int c = s_cnt[q * nk + a.n];
                s_cnt[q * nk + a.n] = at;
                at += c;
            }
            int32_t *seg = a.buf + a.l.seg;
            seg[a.n] = live;
            seg[a.n + 1] = int(a.M);
            seg[a.n + 2 + a.n] = s_all[2];
            seg[a.n + 2 + a.n + 1] = s_all[2];
            a.buf[0] = s_all[1];
            a.buf[1] = s_all[1] + nnt;
            a.buf[2] = s_all[2];
        }
        int4 *tl = reinterpret_cast<int4 *>(a.buf + a.l.tiles) + s_all[1];
        for (int q = t; q < nnt; q += 64 * PLAN_WAVES)
            tl[q] = make_int4(-1, live + q * T, none - q * T < T ? none - q * T : T, 0);
        __syncthreads();
    }
    if (bad && a.err) atomicOr(a.err, BSQ_DEVERR_BAD_SET);
}

// ---------------------------------------------------------------------------
// Shared by the products.
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
    const int32_t *plan;
    PlanLayout l;
    Proj p[BSQ_MAX_GROUP];
    const uint16_t *X;
    const uint16_t *dx0;
    void *dx;
    int64_t M, d_in, ldx, lddx0, lddx;
    int n, np, rank, rp, ksplit;
    int y_bf16, dx_bf16, accumulate;
    float *part;      // [ksplit][np][M][rp]: partial t or u, places in plan order
    uint16_t *hl;     // [2 np][M][3][rp]: s t (then u) as three bf16 parts
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

__device__ __forceinline__ bf16x8_t as_bf16(frag_t v) { return __builtin_bit_cast(bf16x8_t, v); }

__device__ __forceinline__ f32x4_t mfma(frag_t l, frag_t r, f32x4_t c)
{
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16(l), as_bf16(r), c, 0, 0, 0);
}

// Eight values p[0 .. 8) of a row, those from `valid` on as zero. VEC: p is
// 16-byte aligned and valid is 8 or more, or 0 or less.
template <bool VEC>
__device__ __forceinline__ frag_t load8(const uint16_t *p, int64_t valid)
{
    if constexpr (VEC) {
        return valid > 0 ? *reinterpret_cast<const frag_t *>(p) : frag_t{0u, 0u, 0u, 0u};
    } else {
        frag_t v = frag_t{0u, 0u, 0u, 0u};
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (e < valid) v[e >> 1] |= uint32_t(p[e]) << (16 * (e & 1));
        return v;
    }
}

// Eight values stride apart, those from `valid` on as zero.
__device__ __forceinline__ frag_t load8_strided(const uint16_t *p, int64_t stride, int64_t valid)
{
    frag_t v = frag_t{0u, 0u, 0u, 0u};
#pragma unroll
    for (int e = 0; e < 8; ++e)
        if (e < valid) v[e >> 1] |= uint32_t(p[e * stride]) << (16 * (e & 1));
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

// ---------------------------------------------------------------------------
// shrink: part[z][p][place][r] = sum over the block's share of the long
// dimension of W[r][k] S[token][k]; forward S = x and W = A (k contiguous),
// backward S = dy and W = B^T (STRIDED: k apart by the rank).
// 16-token tiles: the four waves share the tile and split k. 64-token tiles: a
// wave per 16 tokens.
// ---------------------------------------------------------------------------
template <int RB, bool BACK, bool VEC, int TG>
__global__ __launch_bounds__(AT) void adapters_shrink(const AdArgs a)
{
    constexpr int U = (RB >= 4) ? 2 : 4;  // 32-deep steps whose loads are in flight together
    if (int(blockIdx.x) >= a.plan[0]) return;
    const int4 tile = reinterpret_cast<const int4 *>(a.plan + a.l.tiles)[blockIdx.x];
    const Proj &p = a.p[blockIdx.z];
    const int t = threadIdx.x, lane = t & 63, g = lane >> 4, r16 = lane & 15;
    const int wave = __builtin_amdgcn_readfirstlane(t >> 6);
    const int64_t K = BACK ? p.d_out : a.d_in;
    const int64_t lds = BACK ? p.ldb : a.ldx;
    const uint16_t *S = BACK ? static_cast<const uint16_t *>(p.base) : a.X;
    const int ad = tile.x, re = rank_of(p, ad, a.rank);
    const uint16_t *W = BACK ? p.B + int64_t(ad) * K * a.rank : p.A + int64_t(ad) * a.rank * K;
    // this wave's range of k, whole steps of 32
    const int64_t nshare = int64_t(a.ksplit) * (TG == 1 ? 4 : 1);
    const int64_t share = int64_t(blockIdx.y) * (TG == 1 ? 4 : 1) + (TG == 1 ? wave : 0);
    const int64_t steps = (K + 31) / 32;
    const int64_t s0 = steps * share / nshare, s1 = steps * (share + 1) / nshare;
    const int tok = (TG == 1 ? 0 : 16 * wave) + r16;
    if (TG != 1 && 16 * wave >= tile.z) return;
    const int place = tile.y + (tok < tile.z ? tok : tile.z - 1);
    const uint16_t *srow = S + int64_t(a.plan[a.l.order + place]) * lds;
    f32x4_t acc[RB];
#pragma unroll
    for (int b = 0; b < RB; ++b) acc[b] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
    for (int64_t s = s0; s < s1; s += U) {
        frag_t x[U], w[U][RB];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int64_t k = 32 * (s + u) + 8 * g, left = (s + u < s1) ? K - k : 0;
            x[u] = load8<VEC>(srow + k, left);
#pragma unroll
            for (int b = 0; b < RB; ++b) {
                const int r = 16 * b + r16;
                const int64_t valid = r < re ? left : 0;
                if constexpr (BACK) w[u][b] = load8_strided(W + k * a.rank + r, a.rank, valid);
                else w[u][b] = load8<VEC>(W + r * K + k, valid);
            }
        }
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int b = 0; b < RB; ++b) acc[b] = mfma(w[u][b], x[u], acc[b]);
    }
    // lane: ranks 16 b + 4 g .. + 3 of token r16
    if constexpr (TG == 1) {
        __shared__ f32x4_t s_acc[4][RB][64];
#pragma unroll
        for (int b = 0; b < RB; ++b) s_acc[wave][b][lane] = acc[b];
        __syncthreads();
        for (int b = wave; b < RB; b += 4) {
            f32x4_t v = s_acc[0][b][lane];
#pragma unroll
            for (int q = 1; q < 4; ++q) v += s_acc[q][b][lane];
            if (tok < tile.z)
                *reinterpret_cast<f32x4_t *>(a.part + ((int64_t(blockIdx.y) * a.np + blockIdx.z) * a.M + place) * a.rp +
                                             16 * b + 4 * g) = v;
        }
    } else {
        if (tok < tile.z)
#pragma unroll
            for (int b = 0; b < RB; ++b)
                *reinterpret_cast<f32x4_t *>(a.part + ((int64_t(blockIdx.y) * a.np + blockIdx.z) * a.M + place) * a.rp +
                                             16 * b + 4 * g) = acc[b];
    }
}

// Sum over the splits, in order, of eight partial values from rank r on.
__device__ __forceinline__ void part_sum(const AdArgs &a, int p, int place, int r, float (&v)[8])
{
    const float *q = a.part + (int64_t(p) * a.M + place) * a.rp + r;
    const int64_t step = int64_t(a.np) * a.M * a.rp;
    f32x4_t x = *reinterpret_cast<const f32x4_t *>(q), y = *reinterpret_cast<const f32x4_t *>(q + 4);
    for (int z = 1; z < a.ksplit; ++z) {
        x += *reinterpret_cast<const f32x4_t *>(q + z * step);
        y += *reinterpret_cast<const f32x4_t *>(q + z * step + 4);
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        v[e] = x[e];
        v[4 + e] = y[e];
    }
}

// ---------------------------------------------------------------------------
// expand: y = y0 + s B t (or dx = dx0 + sum over projections of A^T u).
// A block: a tile and 256 columns; a wave: 16 tokens (64-token tiles) over
// all of them, or 64 columns of all 16. A lane's accumulators are 16
// consecutive columns of one token (W's rows interleave in runs of four), so
// y is read and written in whole 16-byte words.
// ---------------------------------------------------------------------------
constexpr int EXP_COLS = 256;

template <int RB, bool BACK, bool VEC, int TG, bool F32>
__global__ __launch_bounds__(AT) void adapters_expand(const AdArgs a)
{
    if (int(blockIdx.x) >= a.plan[1]) return;
    const int4 tile = reinterpret_cast<const int4 *>(a.plan + a.l.tiles)[blockIdx.x];
    const int t = threadIdx.x, lane = t & 63, g = lane >> 4, r16 = lane & 15;
    const int wave = __builtin_amdgcn_readfirstlane(t >> 6);
    const Proj &pz = a.p[BACK ? 0 : blockIdx.z];
    const int64_t C = BACK ? a.d_in : pz.d_out;
    const int64_t c0 = int64_t(blockIdx.y) * EXP_COLS + (TG == 1 ? 64 * wave : 0);
    const int64_t c1 = (TG == 1) ? c0 + 64 : c0 + EXP_COLS;
    const int tok = (TG == 1 ? 0 : 16 * wave) + r16;
    if (TG != 1 && 16 * wave >= tile.z) return;
    if (c0 >= C) return;
    const void *base = BACK ? static_cast<const void *>(a.dx0) : pz.base;
    void *out = BACK ? a.dx : pz.y;
    const int64_t ldb = BACK ? a.lddx0 : pz.ldb, ldo = BACK ? a.lddx : pz.ldy;
    constexpr bool out_bf16 = !F32, base_bf16 = BACK || !F32;
    const bool live = tok < tile.z;
    const int place = tile.y + (live ? tok : tile.z - 1);
    const int64_t m = a.plan[a.l.order + place];
    const int ad = tile.x;
    if (ad < 0 && base == out) {
        // unchanged rows; t of a token without an adapter is still written below
        if (BACK || !pz.t || blockIdx.y != 0) return;
    }
    // t or u of the lane's token in two parts: lanes g < 2 the first
    const int P0 = BACK ? 0 : int(blockIdx.z), P1 = BACK ? a.np : P0 + 1;
    for (int64_t c = c0; c < c1 && c < C; c += 64) {
        f32x4_t acc[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[j] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
        for (int pi = P0; pi < P1; ++pi) {
            const Proj &p = a.p[pi];
            const int re = ad >= 0 ? rank_of(p, ad, a.rank) : 0;
            const float sc = ad >= 0 ? scale_of(p, ad) : 0.0f;
#pragma unroll
            for (int b = 0; b < RB; ++b) {
                const int r0 = 16 * b + 8 * (g & 1);  // the lane's ranks r0 .. + 7
                // the first part and the second share a product, the third (F32) has its own
                frag_t tf = frag_t{0u, 0u, 0u, 0u}, tf3 = tf;
                if constexpr (BACK) {
                    if (ad >= 0) {
                        const uint16_t *q = a.hl + (int64_t(a.np + pi) * a.M + place) * 3 * a.rp + r0;
                        tf = *reinterpret_cast<const frag_t *>(q + (g >> 1) * a.rp);
                        if (F32 && g < 2) tf3 = *reinterpret_cast<const frag_t *>(q + 2 * a.rp);
                    }
                } else {
                    float v[8] = {0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f};
                    if (ad >= 0) part_sum(a, pi, place, r0, v);
                    if (p.t && blockIdx.y == 0 && c == 0 && live && g < 2)
#pragma unroll
                        for (int e = 0; e < 8; ++e)
                            if (r0 + e < a.rank) p.t[m * a.rank + r0 + e] = v[e];
#pragma unroll
                    for (int e = 0; e < 8; ++e) v[e] *= sc;
                    frag_t part[3];
                    split3(v, part);
                    tf = (g < 2) ? part[0] : part[1];
                    if (F32 && g < 2) tf3 = part[2];
                }
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int64_t cc = c + (r16 >> 2) * 16 + 4 * j + (r16 & 3);
                    const int64_t row = cc < C ? cc : C - 1;
                    frag_t w;
                    if constexpr (BACK) {
                        w = load8_strided(p.A + (int64_t(ad < 0 ? 0 : ad) * a.rank + r0) * C + row, C, re - r0);
                    } else {
                        w = load8<VEC>(p.B + (int64_t(ad < 0 ? 0 : ad) * C + row) * a.rank + r0,
                                       VEC && r0 < re ? 8 : re - r0);
                        // ranks past the adapter's own hold anything
                        if (VEC && p.ranks && re - r0 < 8)
#pragma unroll
                            for (int e = 0; e < 8; ++e)
                                if (e >= re - r0) w[e >> 1] &= (e & 1) ? 0x0000ffffu : 0xffff0000u;
                    }
                    if (F32) acc[j] = mfma(w, tf3, acc[j]);
                    acc[j] = mfma(w, tf, acc[j]);
                }
            }
        }
        // lane: columns c + 16 g .. + 15 of its token
        if (!live) continue;
        const int64_t col = c + 16 * g;
        if (col >= C) continue;
        const int64_t nc = C - col < 16 ? C - col : 16;
        float v[16];
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int r = 0; r < 4; ++r) v[4 * j + r] = acc[j][r];
        const bool whole = VEC && nc == 16;
        if (base) {
            if (base_bf16) {
                const uint16_t *q = static_cast<const uint16_t *>(base) + m * ldb + col;
                if (whole) {
                    const frag_t w[2] = {reinterpret_cast<const frag_t *>(q)[0], reinterpret_cast<const frag_t *>(q)[1]};
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        v[2 * e] += __uint_as_float(w[e >> 2][e & 3] << 16);
                        v[2 * e + 1] += __uint_as_float(w[e >> 2][e & 3] & 0xffff0000u);
                    }
                } else {
#pragma unroll
                    for (int e = 0; e < 16; ++e)
                        if (e < nc) v[e] += bf16_to_f32(q[e]);
                }
            } else {
                const float *q = static_cast<const float *>(base) + m * ldb + col;
                if (whole) {
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const f32x4_t w = reinterpret_cast<const f32x4_t *>(q)[j];
#pragma unroll
                        for (int r = 0; r < 4; ++r) v[4 * j + r] += w[r];
                    }
                } else {
#pragma unroll
                    for (int e = 0; e < 16; ++e)
                        if (e < nc) v[e] += q[e];
                }
            }
        }
        if (out_bf16) {
            uint16_t *q = static_cast<uint16_t *>(out) + m * ldo + col;
            if (whole) {
                frag_t w[2];
#pragma unroll
                for (int e = 0; e < 8; ++e) w[e >> 2][e & 3] = pack_bf16x2(v[2 * e], v[2 * e + 1]);
                reinterpret_cast<frag_t *>(q)[0] = w[0];
                reinterpret_cast<frag_t *>(q)[1] = w[1];
            } else {
#pragma unroll
                for (int e = 0; e < 16; ++e)
                    if (e < nc) q[e] = f32_to_bf16(v[e]);
            }
        } else {
            float *q = static_cast<float *>(out) + m * ldo + col;
            if (whole) {
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    reinterpret_cast<f32x4_t *>(q)[j] = f32x4_t{v[4 * j], v[4 * j + 1], v[4 * j + 2], v[4 * j + 3]};
            } else {
#pragma unroll
                for (int e = 0; e < 16; ++e)
                    if (e < nc) q[e] = v[e];
            }
        }
    }
}

// ---------------------------------------------------------------------------
// Backward: s t and u in three bf16 parts, in plan order, zero past an adapter's
// rank. One thread per eight ranks of a token; z: projection.
// ---------------------------------------------------------------------------
__global__ __launch_bounds__(AT) void adapters_parts(const AdArgs a)
{
    const int groups = a.rp / 8;
    const int64_t i = int64_t(blockIdx.x) * AT + threadIdx.x;
    const int64_t place = i / groups;
    const int r0 = int(i - place * groups) * 8;
    const int32_t *seg = a.plan + a.l.seg;
    if (place >= seg[a.n]) return;
    // its adapter: the last whose first place is not past it
    int lo = 0, hi = a.n;
    while (hi - lo > 1) {
        const int mid = (lo + hi) / 2;
        if (seg[mid] <= place) lo = mid;
        else hi = mid;
    }
    const int ad = lo, pi = blockIdx.z;
    const Proj &p = a.p[pi];
    const int re = rank_of(p, ad, a.rank);
    const float sc = scale_of(p, ad);
    const int64_t m = a.plan[a.l.order + place];
    float v[8];
    frag_t part[3];
#pragma unroll
    for (int h = 0; h < 2; ++h) {  // s t, then u
        if (h == 1) part_sum(a, pi, int(place), r0, v);
#pragma unroll
        for (int e = 0; e < 8; ++e)
            v[e] = (r0 + e < re) ? sc * (h == 0 ? p.t[m * a.rank + r0 + e] : v[e]) : 0.0f;
        split3(v, part);
        uint16_t *q = a.hl + (int64_t(h * a.np + pi) * a.M + place) * 3 * a.rp + r0;
#pragma unroll
        for (int k = 0; k < 3; ++k) *reinterpret_cast<frag_t *>(q + k * a.rp) = part[k];
    }
}

// ---------------------------------------------------------------------------
// outer: of a piece's tokens, G[c][r] = sum_m S[m][c] Q[m][r]: dB (S = dy, Q =
// s t) or dA transposed (S = x, Q = u). A wave owns 64 columns. Per step of 32
// tokens it stages its 32 x 64 of S in LDS and the block stages Q's three parts;
// both are read transposed, as operands with the tokens along the product's
// depth. blockIdx.z: 2 projection + (1 for dA).
//
// LDS rows of S: 64 columns, 128 bytes, in 32-byte groups; group q of row k
// lies at q ^ key(k), so that the eight rows that half a wave reads together
// fall on different banks.
// ---------------------------------------------------------------------------
constexpr int OUT_COLS = 256;

typedef short s16x4_t __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) s16x4_t lds_s16x4_t;

// 8 tokens (rows k0 .. k0 + 7 of 16-column groups) of the lane's column: two
// transposed reads of four rows. p: the lane's own 8 bytes of the first row
// group (row 8 g + r16 / 4, columns 4 (r16 % 4) ..), four: bytes of four rows.
__device__ __forceinline__ frag_t read_tr(const uint8_t *p, int four)
{
    typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
    const u32x2 a = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_t *)p));
    const u32x2 b = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_t *)(p + four)));
    return frag_t{a[0], a[1], b[0], b[1]};
}

template <int RB, bool VEC>
__global__ __launch_bounds__(AT) void adapters_outer(const AdArgs a)
{
    __shared__ __attribute__((aligned(16))) uint8_t s_s[4][32 * 128];
    __shared__ __attribute__((aligned(16))) uint8_t s_q[32 * 3 * RB * 32];  // [32][3][16 RB] bf16
    if (int(blockIdx.x) >= a.plan[2]) return;
    const int4 piece = reinterpret_cast<const int4 *>(a.plan + a.l.pieces)[blockIdx.x];
    const int pi = int(blockIdx.z) >> 1, is_a = int(blockIdx.z) & 1;
    const Proj &p = a.p[pi];
    const int64_t C = is_a ? a.d_in : p.d_out;
    const int64_t cb = int64_t(blockIdx.y) * OUT_COLS;
    if (cb >= C) return;
    const int t = threadIdx.x, lane = t & 63, g = lane >> 4, r16 = lane & 15;
    const int wave = __builtin_amdgcn_readfirstlane(t >> 6);
    const int64_t c0 = cb + 64 * wave;
    const uint16_t *S = is_a ? a.X : static_cast<const uint16_t *>(p.base);
    const int64_t lds = is_a ? a.ldx : p.ldb;
    const uint16_t *Q = a.hl + (int64_t(is_a ? a.np + pi : pi) * a.M + piece.y) * 3 * a.rp;
    const int32_t *order = a.plan + a.l.order + piece.y;
    f32x4_t acc[4][RB];
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int b = 0; b < RB; ++b) acc[i][b] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
    uint8_t *ss = s_s[wave];
    // staging: lane -> row lane / 8 (+ 8 i), columns 8 (lane % 8) ..
    const int64_t sc = c0 + 8 * (lane & 7);
    constexpr int QW = 6 * RB, QV = (32 * QW + AT - 1) / AT;  // 16-byte words of a row of Q, and per thread
    frag_t sv[4], qv[QV];
    auto fetch = [&](int k0) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int k = k0 + 8 * i + (lane >> 3);
            const bool in = k < piece.z;
            const int64_t m = order[in ? k : 0];
            sv[i] = load8<VEC>(S + m * lds + sc, in ? C - sc : 0);
        }
#pragma unroll
        for (int q = 0; q < QV; ++q) {
            const int w = t + AT * q, row = w / QW;
            const bool in = row < 32 && k0 + row < piece.z;
            qv[q] = in ? reinterpret_cast<const frag_t *>(Q + int64_t(k0) * 3 * a.rp)[w] : frag_t{0u, 0u, 0u, 0u};
        }
    };
    fetch(0);
    // the lane's row in a transposed read: 8 g + r16 / 4 (+ 4)
    const int kr = 8 * g + (r16 >> 2), key = ((kr >> 1) & 1) | (((kr >> 3) & 1) << 1);
    for (int k0 = 0; k0 < piece.z; k0 += 32) {
        __syncthreads();  // the last step's reads are over
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int k = 8 * i + (lane >> 3), kk = ((k >> 1) & 1) | (((k >> 3) & 1) << 1);
            *reinterpret_cast<frag_t *>(ss + k * 128 + ((((lane & 7) >> 1) ^ kk) << 5) + ((lane & 1) << 4)) = sv[i];
        }
#pragma unroll
        for (int q = 0; q < QV; ++q)
            if (t + AT * q < 32 * QW) reinterpret_cast<frag_t *>(s_q)[t + AT * q] = qv[q];
        __syncthreads();
        if (k0 + 32 < piece.z) fetch(k0 + 32);
        frag_t sf[4];
#pragma unroll
        for (int i = 0; i < 4; ++i)
            sf[i] = read_tr(ss + kr * 128 + ((i ^ key) << 5) + ((r16 & 3) << 3), 4 * 128);
#pragma unroll
        for (int b = 0; b < RB; ++b)
#pragma unroll
            for (int h = 0; h < 3; ++h) {
                const frag_t qf = read_tr(s_q + kr * (96 * RB) + h * (32 * RB) + b * 32 + ((r16 & 3) << 3), 4 * 96 * RB);
#pragma unroll
                for (int i = 0; i < 4; ++i) acc[i][b] = mfma(sf[i], qf, acc[i][b]);
            }
    }
    // lane: columns c0 + 16 i + 4 g .. + 3 at rank 16 b + r16
    const int64_t R = a.rank;
    float *out;
    bool add = false;
    if (piece.w < 0) {
        out = is_a ? p.dA : p.dB;
        out += int64_t(piece.x) * R * C;
        add = a.accumulate;
    } else {
        out = a.slots + int64_t(piece.w) * a.slot_floats;
        for (int q = 0; q < pi; ++q) out += R * (a.p[q].d_out + a.d_in);
        out += is_a ? R * p.d_out : 0;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int b = 0; b < RB; ++b) {
            const int64_t r = 16 * b + r16, c = c0 + 16 * i + 4 * g;
            if (r >= R) continue;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                if (c + e >= C) break;
                float *q = is_a ? out + r * C + c + e : out + (c + e) * R + r;
                *q = add ? *q + acc[i][b][e] : acc[i][b][e];
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
    size_t part, hl, slots, total;
    int64_t slot_floats;
};

// Ranks of a row of t in the workspace: one, two, four or eight blocks of 16.
int rank_pad(int rank) { return rank <= 16 ? 16 : (rank <= 32 ? 32 : (rank <= 64 ? 64 : 128)); }

// Splits of a shrink's long dimension (the longest of the group): until the
// launch has about 2048 blocks, each wave keeping 128 or more of it.
int shrink_splits(int64_t tiles, int np, int64_t K, bool split_waves)
{
    const int64_t most = std::max<int64_t>(1, K / (split_waves ? 512 : 128));
    return int(std::clamp<int64_t>(2048 / std::max<int64_t>(1, tiles * np), 1, std::min<int64_t>(most, 8)));
}

AdLayout ad_layout(bool back, int64_t M, int64_t n, int np, int rank, int64_t d_in, const int64_t *d_out)
{
    const PlanLayout pl = plan_layout(M, n);
    AdLayout l{};
    int64_t longest = back ? 0 : d_in;
    for (int i = 0; i < np; ++i) {
        if (back) longest = std::max(longest, d_out[i]);
        l.slot_floats += int64_t(rank) * (d_in + d_out[i]);
    }
    l.slot_floats = (l.slot_floats + 3) / 4 * 4;
    l.ksplit = shrink_splits(M / pl.tile + 1, np, longest, pl.tile == 16);
    const size_t rp = size_t(rank_pad(rank));
    l.part = 0;
    l.hl = l.part + align256(size_t(l.ksplit) * np * size_t(M) * rp * 4);
    l.slots = l.hl + (back ? align256(size_t(2 * np) * size_t(M) * 3 * rp * 2) : 0);
    l.total = l.slots + (back ? align256(size_t(pl.max_slots) * size_t(l.slot_floats) * 4) : 0);
    return l;
}

template <bool VEC, int TG>
hipError_t shrink_expand(const AdArgs &a, bool back, bool second, dim3 grid, hipStream_t st)
{
#define BSQ_RB(RB)                                                                                                   \
    case RB:                                                                                                         \
        if (!second && back) hipLaunchKernelGGL((adapters_shrink<RB, true, VEC, TG>), grid, dim3(AT), 0, st, a);     \
        else if (!second) hipLaunchKernelGGL((adapters_shrink<RB, false, VEC, TG>), grid, dim3(AT), 0, st, a);       \
        else if (back && a.dx_bf16) hipLaunchKernelGGL((adapters_expand<RB, true, VEC, TG, false>), grid, dim3(AT), 0, st, a); \
        else if (back) hipLaunchKernelGGL((adapters_expand<RB, true, VEC, TG, true>), grid, dim3(AT), 0, st, a);     \
        else if (a.y_bf16) hipLaunchKernelGGL((adapters_expand<RB, false, VEC, TG, false>), grid, dim3(AT), 0, st, a); \
        else hipLaunchKernelGGL((adapters_expand<RB, false, VEC, TG, true>), grid, dim3(AT), 0, st, a);              \
        break;
    switch (a.rp / 16) {
        BSQ_RB(1)
        BSQ_RB(2)
        BSQ_RB(4)
        BSQ_RB(8)
    }
#undef BSQ_RB
    return hipGetLastError();
}

hipError_t shrink_expand(const AdArgs &a, bool back, bool second, bool vec, dim3 grid, hipStream_t st)
{
    const bool tg1 = a.l.tile == 16;
    if (vec) return tg1 ? shrink_expand<true, 1>(a, back, second, grid, st) : shrink_expand<true, 4>(a, back, second, grid, st);
    return tg1 ? shrink_expand<false, 1>(a, back, second, grid, st) : shrink_expand<false, 4>(a, back, second, grid, st);
}

template <bool VEC>
hipError_t launch_outer(const AdArgs &a, dim3 grid, hipStream_t st)
{
    const int rb = a.rp / 16;
    if (rb == 1) hipLaunchKernelGGL((adapters_outer<1, VEC>), grid, dim3(AT), 0, st, a);
    else if (rb == 2) hipLaunchKernelGGL((adapters_outer<2, VEC>), grid, dim3(AT), 0, st, a);
    else if (rb == 4) hipLaunchKernelGGL((adapters_outer<4, VEC>), grid, dim3(AT), 0, st, a);
    else hipLaunchKernelGGL((adapters_outer<8, VEC>), grid, dim3(AT), 0, st, a);
    return hipGetLastError();
}

bool al16(const void *p, int64_t row_bytes) { return ((reinterpret_cast<uintptr_t>(p) | uintptr_t(row_bytes)) & 15) == 0; }

}  // namespace

int64_t adapters_tile(int64_t M) { return M <= 1024 ? 16 : 64; }

size_t adapters_plan_bytes(int64_t M, int64_t n) { return size_t(plan_layout(M, n).words) * 4; }

hipError_t launch_adapters_plan(const int32_t *ids, int64_t M, int64_t n, void *buf, int32_t *err, hipStream_t st)
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
    if (lds > 60 * 1024) {
        const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void *>(&adapters_plan_kernel),
                                                 hipFuncAttributeMaxDynamicSharedMemorySize, int(lds));
        if (e != hipSuccess) return e;
    }
    hipLaunchKernelGGL(adapters_plan_kernel, dim3(1), dim3(64 * PLAN_WAVES), lds, st, a);
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
    a.M = c.plan->M;
    a.n = c.plan->n;
    a.l = plan_layout(a.M, a.n);
    int64_t d_out[BSQ_MAX_GROUP], most = 0;
    for (int i = 0; i < c.np; ++i) most = std::max(most, d_out[i] = c.pools[i].d_out);
    const AdLayout l = ad_layout(back, a.M, a.n, c.np, c.rank, c.d_in, d_out);
    char *ws = static_cast<char *>(c.ws);
    a.X = static_cast<const uint16_t *>(c.X);
    a.ldx = c.ldx;
    a.d_in = c.d_in;
    a.np = c.np;
    a.rank = c.rank;
    a.rp = rank_pad(c.rank);
    a.ksplit = l.ksplit;
    a.part = reinterpret_cast<float *>(ws + l.part);
    a.hl = reinterpret_cast<uint16_t *>(ws + l.hl);
    a.slots = reinterpret_cast<float *>(ws + l.slots);
    a.slot_floats = l.slot_floats;
    a.y_bf16 = c.y_dtype == BSQ_BF16;
    a.accumulate = c.accumulate;
    const int64_t es = a.y_bf16 ? 2 : 4;
    const bool vx = al16(c.X, 2 * c.ldx) && c.d_in % 8 == 0;
    bool va = vx, vy = c.rank % 8 == 0, vd = true;  // vector loads of x with A, of y with B, of dy
    for (int i = 0; i < c.np; ++i) {
        const bsq_adapter_pool &q = c.pools[i];
        Proj &p = a.p[i];
        p.A = q.A;
        p.B = q.B;
        p.scale = q.scale;
        p.ranks = q.ranks;
        p.d_out = q.d_out;
        p.t = c.t ? c.t[i] : nullptr;
        va = va && al16(q.A, 2 * c.d_in);
        if (back) {
            p.base = c.dy[i];
            p.ldb = c.lddy[i];
            p.dA = c.dA[i];
            p.dB = c.dB[i];
            vd = vd && al16(p.base, 2 * p.ldb) && p.d_out % 8 == 0;
        } else {
            p.base = c.y0 ? c.y0[i] : nullptr;
            p.ldb = c.y0 ? c.ldy0[i] : 0;
            p.y = c.y[i];
            p.ldy = c.ldy[i];
            vy = vy && al16(q.B, 0) && al16(p.base, es * p.ldb) && al16(p.y, es * p.ldy);
        }
    }
    const dim3 sgrid(unsigned(a.l.max_tiles), unsigned(l.ksplit), unsigned(c.np));
    hipError_t e = shrink_expand(a, back, false, back ? vd : va, sgrid, st);
    if (e != hipSuccess) return e;
    if (!back)
        return shrink_expand(a, false, true, vy, dim3(unsigned(a.l.max_tiles), unsigned((most + EXP_COLS - 1) / EXP_COLS), unsigned(c.np)), st);
    hipLaunchKernelGGL(adapters_parts, dim3(unsigned((a.M * (a.rp / 8) + AT - 1) / AT), 1, unsigned(c.np)), dim3(AT), 0, st, a);
    if ((e = hipGetLastError()) != hipSuccess) return e;
    const int64_t widest = std::max(most, c.d_in);
    const dim3 ogrid(unsigned(a.l.max_pieces), unsigned((widest + OUT_COLS - 1) / OUT_COLS), unsigned(2 * c.np));
    e = (vx && vd) ? launch_outer<true>(a, ogrid, st) : launch_outer<false>(a, ogrid, st);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(adapters_pieces, dim3(unsigned((int64_t(c.rank) * widest + 4 * AT - 1) / (4 * AT)), unsigned(a.n), unsigned(2 * c.np)),
                       dim3(AT), 0, st, a);
    if ((e = hipGetLastError()) != hipSuccess || !c.dx) return e;
    a.dx0 = static_cast<const uint16_t *>(c.dx0);
    a.dx = c.dx;
    a.lddx0 = c.lddx0;
    a.lddx = c.lddx;
    a.dx_bf16 = c.dx_dtype == BSQ_BF16;
    const bool vdx = al16(c.dx0, 2 * c.lddx0) && al16(c.dx, (a.dx_bf16 ? 2 : 4) * c.lddx);
    return shrink_expand(a, true, true, vdx, dim3(unsigned(a.l.max_tiles), unsigned((c.d_in + EXP_COLS - 1) / EXP_COLS), 1), st);
}

}  // namespace bsq
