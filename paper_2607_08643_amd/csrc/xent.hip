// Softmax cross entropy of a large vocabulary from hidden states H [T][D] and
// head weights V [N][D], and its gradient, without keeping the T x N logits:
//   z = H V^T,  lse = log sum exp(z),  loss = lse - z_target,
//   d = g (exp(z - lse) - onehot),  dH = d V,  dV = d^T H.
//
// loss: one matrix product whose tiles are reduced where they are made: per
// token and tile the largest logit and the sum of exponentials against it, and
// the target's logit; a second launch joins a token's tiles. 2 T N D
// operations, D-deep; V is read once.
//
// gradient: the vocabulary in pieces of `vp` words. Per piece the logits are
// made again and leave the tile as d in bf16 (the workspace holds one piece; for
// a dV of 32 bits in two bf16 parts, which its product takes one after the other);
// two further products read them: dV's rows of the piece, and the piece's
// contribution to dH, added in fp32 over the pieces in order.
//
// Bound by the matrix cores from some hundred tokens on: 4096 tokens of 151936
// words, 4096 inputs: logits 4.5 ms (1.14 PFLOP/s), dH 3.9 (1.31), dV 4.5 (1.13; the
// whole gradient 12.8, with a dV of 32 bits 17.7); the loss alone of 2000 tokens 2.25
// ms a pass (1.11; 2.37 in a profiled run). One token's loss is one reading of V: 247
// us, 5.0 TB/s.
//
// Tokens without a loss are taken out first: the rows that have one are copied
// next to each other (padded with zeros to whole tiles and to a multiple of
// 64 inputs), and every product runs over those alone.
#include <algorithm>
#include <atomic>
#include <numeric>
#include <type_traits>

#include "gemm_common.h"

namespace bsq {
namespace {

constexpr int XT = 256;
constexpr int VBLK = 256;              // words of a logits tile
constexpr int64_t ROW_PAD = 256;       // token rows are padded to this
constexpr float LOG2E = 1.4426950408889634f;
// Up to this many tokens the tiles are chosen by those that have a loss. Past it,
// 256-token tiles fill the compute units where most tokens have one; where few do
// they do not, nor do dH's splits, which follow all tokens (4096 tokens of which 410
// have a loss, 4096 inputs: 32 blocks of dH).
constexpr int64_t HALF_TOKENS = 1024;

constexpr int ZEROS = 4;

// EPI_DV2: EPI_DV from both parts of d
enum { EPI_STATS, EPI_PROB, EPI_DV, EPI_DV2, EPI_DH };

struct XArgs {
    // header words: 0: tokens with a loss; ZEROS .. + 3: 16 bytes of zeros
    int32_t *hdr, *rows, *pos;    // rows [Tp]: token of a compact row; pos [T]: compact row of a token or -1
    const uint16_t *H, *V;
    int64_t ldh, ldv, T, N, D, Tp, Dp;
    const int64_t *target;
    const float *lse_in, *g_in;
    int32_t *err;
    uint16_t *Hc;                 // [Tp][Dp]
    int32_t *tgt;                 // [Tp] compact targets
    float *lse, *g;               // [Tp] compact
    float2 *stat;                 // [word tiles][Tp]: largest logit, sum of exp against it
    float *ztgt;                  // [Tp]
    float *loss_out, *lse_out;
    // a piece of the vocabulary: words [v0, v0 + vp)
    int64_t v0, vp, dsp;          // dsp: row length of dS
    uint16_t *dS;                 // [Tp][dsp]: d rounded; from column lo on, where that is not 0, what remains
    int64_t lo;
    float *dHp;                   // [hsplit][Tp][Dp]
    int hsplit, first;
    uint16_t *dH;
    void *dV;
    int64_t lddh, lddv;
    int dv_bf16, dv_vec, dh_vec, accumulate;
};

// ---------------------------------------------------------------------------
// The rows that have a loss, in order, and their copies. Up to ROWS_ONE tokens
// every block of the copy finds its rows itself; beyond that one block lists
// them first.
// ---------------------------------------------------------------------------
constexpr int XR = 1024;
constexpr int64_t ROWS_ONE = XR;

// Of XR tokens from m0 on: is the thread's one with a loss, and how many are
// before it; `all` are added up. (Two barriers.)
__device__ __forceinline__ bool count_rows(const XArgs &a, int64_t m0, int &before, int &all, bool &bad, int *s_w)
{
    const int t = threadIdx.x, lane = t & 63, w = t >> 6;
    const int64_t m = m0 + t;
    const int64_t y = m < a.T ? a.target[m] : -1;
    const bool live = y >= 0 && y < a.N;
    bad = y >= a.N;
    const uint64_t bal = __ballot(live);
    if (lane == 0) s_w[w] = __popcll(bal);
    __syncthreads();
    before = __popcll(bal & ((uint64_t(1) << lane) - 1));
    all = 0;
#pragma unroll
    for (int k = 0; k < XR / 64; ++k) {
        before += (k < w) ? s_w[k] : 0;
        all += s_w[k];
    }
    __syncthreads();
    return live;
}

__global__ __launch_bounds__(XR) void xent_rows_kernel(const XArgs a)
{
    __shared__ int s_w[XR / 64];
    int base = 0;
    for (int64_t m0 = 0; m0 < a.T; m0 += XR) {
        const int64_t m = m0 + threadIdx.x;
        int before, all;
        bool bad;
        const bool live = count_rows(a, m0, before, all, bad, s_w);
        if (m < a.T) a.pos[m] = live ? base + before : -1;
        if (live) a.rows[base + before] = int32_t(m);
        if (bad && a.err) atomicOr(a.err, BSQ_DEVERR_BAD_SET);
        base += all;
    }
    if (threadIdx.x == 0) a.hdr[0] = base;
}

// Four compact rows a block, 256 threads each: the hidden state padded with
// zeros, the target, lse and g.
template <bool ONE>
__global__ __launch_bounds__(XR) void xent_pack_kernel(const XArgs a)
{
    __shared__ int s_w[XR / 64], s_row[XR / XT];
    const int t = threadIdx.x, sub = t / XT, tt = t % XT;
    const int64_t first = int64_t(blockIdx.x) * (XR / XT), i = first + sub;
    int64_t m = -1;
    if (blockIdx.x == 0 && t < 4) a.hdr[ZEROS + t] = 0;
    if constexpr (ONE) {
        if (t < XR / XT) s_row[t] = -1;
        int before, all;
        bool bad;
        const bool live = count_rows(a, 0, before, all, bad, s_w);
        if (live && before >= first && before < first + XR / XT) s_row[before - first] = t;
        if (blockIdx.x == 0) {
            if (t < a.T) a.pos[t] = live ? before : -1;
            if (bad && a.err) atomicOr(a.err, BSQ_DEVERR_BAD_SET);
            if (t == 0) a.hdr[0] = all;
        }
        __syncthreads();
        m = s_row[sub];
    } else {
        m = (i < a.hdr[0]) ? a.rows[i] : -1;
    }
    const uint16_t *src = a.H + (m < 0 ? 0 : m) * a.ldh;
    uint16_t *dst = a.Hc + i * a.Dp;
    const bool vec = ((reinterpret_cast<uintptr_t>(a.H) | uintptr_t(2 * a.ldh)) & 15) == 0;
    for (int64_t c = 8 * tt; c < a.Dp; c += 8 * XT) {
        u32x4_t v = u32x4_t{0u, 0u, 0u, 0u};
        if (m >= 0 && c < a.D) {  // (D is a multiple of 8)
            if (vec) v = *reinterpret_cast<const u32x4_t *>(src + c);
            else
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e >> 1] |= uint32_t(src[c + e]) << (16 * (e & 1));
        }
        *reinterpret_cast<u32x4_t *>(dst + c) = v;
    }
    if (tt == 0) {
        a.tgt[i] = m >= 0 ? int32_t(a.target[m]) : -1;
        if (a.g) {
            a.g[i] = m >= 0 ? a.g_in[m] : 0.0f;
            a.lse[i] = m >= 0 ? a.lse_in[m] : 0.0f;
        }
    }
}

// ---------------------------------------------------------------------------
// The products. Out[left][right] = sum_k L[left][k] R[right][k]; WM x WN
// waves, a wave owns MF groups of 16 right rows (tokens; dV: words) and NF
// groups of 16 left rows (words; dV, dH: inputs). Steps of 32 deep reach a ring
// of NS LDS slots by DMA, NS steps ahead; the fragments of step u + 1 are read
// while the products of step u issue.
//
// An operand lies in memory either with k contiguous (logits: H, V; dH: d) or
// with k as its row (dH: V; dV: d and H), and is staged as it lies:
//   k contiguous: slot rows of 32 k (64 bytes, four 16-byte chunks); chunk c of
//     row r lies at c ^ key, key = -(r / 4) % 4 (left operand of the logits, whose
//     fragments take rows in runs of four: -(r / 4 NF) % 4). A 16-byte LDS read
//     serves lanes 0-3, 12-15 and 20-27 of a half wave together, then the others:
//     with this key each of those sets falls on all 64 banks once (with
//     (r / 4) % 4 the counters showed two accesses per bank);
//   k as row (256 columns): blocks of eight k, k % 4 + 4 (k / 8 % 2) their rows, as
//     [pair of 16-column groups][row][64 bytes]; the two groups change places in
//     rows 4 to 7. A fragment is read transposed, four k of 16 columns at a time:
//     half a wave takes the eight rows of one block together, 32 bytes of each, on
//     all banks once, and the next pair of groups is a constant further on.
// ---------------------------------------------------------------------------
template <int MF, int NF, int WM, int WN>
struct XShape {
    static constexpr int NW = WM * WN;
    static constexpr int RU = MF * WM, LU = NF * WN;
    static constexpr int BR = 16 * RU, BL = 16 * LU;
    static constexpr int SLOT = (RU + LU) * 1024;
    static constexpr int NS_FIT = GEMM_LDS_BYTES / SLOT;
    static constexpr int NS = NS_FIT < 8 ? NS_FIT : 8;
    static constexpr int NI = RU + LU;
    static constexpr int PMAX = (NI + NW - 1) / NW, PMIN = NI / NW;
    static constexpr size_t LDS = size_t(NS) * SLOT;
    static_assert(NS >= 3, "two steps in flight beside the one being read");
    static_assert((NS - 1) * PMAX <= 63, "wait count fits vmcnt");
    static_assert(WM * BL * 8 <= int(LDS) && WN * BR * 8 <= int(LDS), "statistics fit the ring");
};

typedef short s16x4_t __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) s16x4_t lds_s16x4_t;

// Two transposed reads, of four k rows each: eight k of the lane's column. The
// pointers are restrict so that the reads carry alias information: without any,
// the compiler waits for every DMA in flight ahead of each (the gradient's
// products took 1.31 ms instead of 1.0). The waits that are needed are in the
// loop, as for the plain reads.
__device__ __forceinline__ bf16x8_t read_tr(const uint8_t *__restrict p, const uint8_t *__restrict q)
{
    const s16x4_t x = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_t *)p);
    const s16x4_t y = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_t *)q);
    return __builtin_bit_cast(bf16x8_t, __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7));
}

// Largest value and sum of exponentials against it, joined with another pair.
// (A pair of no values is -inf and 0.)
__device__ __forceinline__ void join_stats(float &m, float &s, float m2, float s2)
{
    const float mm = m2 > m ? m2 : m;
    const float ref = (mm == -__builtin_inff()) ? 0.0f : mm;
    s = s * __builtin_amdgcn_exp2f((m - ref) * LOG2E) + s2 * __builtin_amdgcn_exp2f((m2 - ref) * LOG2E);
    m = mm;
}

// Tiles of a product over `live` tokens, and splits of dH's depth: until the
// launch fills the compute units.
struct XTiles {
    int rt, lt, splits;
};

template <int EPI, int BR, int BL>
__device__ __forceinline__ XTiles xent_tiles(const XArgs &a, int live)
{
    const int64_t rrows = (EPI == EPI_DV || EPI == EPI_DV2) ? a.vp : live;
    const int64_t lrows = (EPI == EPI_STATS || EPI == EPI_PROB) ? a.vp : a.D;
    XTiles n{int((rrows + BR - 1) / BR), int((lrows + BL - 1) / BL), 1};
    if (EPI == EPI_DH) {
        const int fill = n.rt > 0 ? 256 / (n.rt * n.lt) : 1;
        n.splits = fill < 1 ? 1 : (fill < a.hsplit ? fill : a.hsplit);
    }
    return n;
}

// Whether 128-token tiles finish before 256-token ones: rounds of tiles over the
// 256 compute units, of 2/3 the time (512 tokens of 32003 words: 168 us in two
// rounds, 129 in one; 301 tokens of which 180 have a loss: 98 in one, 122).
template <int EPI>
__device__ __forceinline__ bool xent_half_tiles(const XArgs &a, int live)
{
    const XTiles h = xent_tiles<EPI, 128, 256>(a, live), w = xent_tiles<EPI, 256, 256>(a, live);
    const int rh = (h.rt * h.lt * h.splits + 255) / 256, rw = (w.rt * w.lt * w.splits + 255) / 256;
    return 2 * rh * w.splits < 3 * rw * h.splits;
}

template <int EPI, int MF, int NF, int WM, int WN>
__device__ __forceinline__ void xent_tile(const XArgs &a, int live)
{
    using G = XShape<MF, NF, WM, WN>;
    constexpr bool LOGITS = EPI == EPI_STATS || EPI == EPI_PROB;
    constexpr bool DV = EPI == EPI_DV || EPI == EPI_DV2;
    constexpr int PARTS = (EPI == EPI_DV2) ? 2 : 1;  // of d, one after the other along k
    constexpr bool LK = LOGITS;              // left operand k contiguous
    constexpr bool RK = !DV;                 // right operand k contiguous
    static_assert((LK || G::LU == 16) && (RK || G::RU == 16), "256 columns where k is the row");
    constexpr int LSH = (NF == 4) ? 4 : (NF == 2 ? 3 : 2);  // log2(4 NF)
    extern __shared__ __attribute__((aligned(16))) uint4 s_mem4[];
    uint8_t *s_mem = reinterpret_cast<uint8_t *>(s_mem4);
    const int t = threadIdx.x, lane = t & 63, g = lane >> 4, r16 = lane & 15;
    const int wave = __builtin_amdgcn_readfirstlane(t >> 6);
    const int wm = wave / WN, wn = wave % WN;

    // Tiles: right tiles x left tiles (x splits of k for dH); every XCD takes a
    // run of them that walks up to 8 right tiles before the next left one.
    const XTiles n = xent_tiles<EPI, G::BR, G::BL>(a, live);
    const int rt = n.rt, lt = n.lt, splits = n.splits, total = rt * lt * splits;
    if (int(blockIdx.x) >= total) return;
    const int xcd = blockIdx.x & 7, per = total >> 3, rem = total & 7;
    int lg = xcd * per + (xcd < rem ? xcd : rem) + int(blockIdx.x >> 3);
    const int z = lg / (rt * lt);
    lg -= z * (rt * lt);
    const int band = lg / (8 * lt);
    lg -= band * 8 * lt;
    const int bh = (rt - 8 * band < 8) ? rt - 8 * band : 8;
    const int by = 8 * band + lg % bh, bx = lg / bh;

    // k: steps of 32, an even number; valid up to kmax (of a part)
    const int64_t kmax = LOGITS ? a.D : (DV ? live : (a.N - a.v0 < a.vp ? a.N - a.v0 : a.vp));
    const int part = 2 * int((kmax + 63) / 64), pairs = PARTS * part / 2;
    const int kb = 2 * int(int64_t(pairs) * z / splits), ke = 2 * int(int64_t(pairs) * (z + 1) / splits);
    const int ku = ke - kb;

    const uint16_t *L = LOGITS ? a.V + a.v0 * a.ldv : (DV ? a.Hc : a.V + a.v0 * a.ldv);
    const int64_t ldl = LOGITS ? a.ldv : (DV ? a.Dp : a.ldv);
    const uint16_t *R = LOGITS ? a.Hc : a.dS;
    const int64_t ldr = LOGITS ? a.Dp : a.dsp;
    // rows (columns, k as row) that exist: those past them are read from the last
    const int64_t lend = LOGITS ? (a.N - a.v0) : a.D;

    // DMA: unit v of a step is one instruction of the wave, 16 bytes a lane.
    const uint16_t *src[G::PMAX];
    int kof[G::PMAX];      // k (contiguous: of the lane's chunk; as row: of its row) within the step
#pragma unroll
    for (int r = 0; r < G::PMAX; ++r) {
        const int v0 = wave + G::NW * r, v = (v0 < G::NI) ? v0 : G::NI - 1;
        const bool right = v < G::RU;
        const int u = right ? v : v - G::RU;
        const uint16_t *mat = right ? R : L;
        const int64_t ld = right ? ldr : ldl, tile0 = right ? int64_t(by) * G::BR : int64_t(bx) * G::BL;
        if (right ? RK : LK) {
            const int row = 16 * u + (lane >> 2);
            const int key = -(row >> (right ? 2 : LSH)) & 3;
            kof[r] = 8 * ((lane & 3) ^ key);
            int64_t at = tile0 + row;
            if (!right && at >= lend) at = lend - 1;
            src[r] = mat + at * ld + kof[r];
        } else {
            const int blk = u >> 2, key = (lane >> 2) & 7, chunk = lane & 3;
            const int k = 16 * (blk >> 1) + 8 * (key >> 2) + 4 * (blk & 1) + (key & 3);
            int64_t col = tile0 + 32 * (2 * (u & 3) + (lane >> 5)) + 16 * ((chunk >> 1) ^ (key >> 2)) + 8 * (chunk & 1);
            if (!right && col >= lend) col = 0;
            kof[r] = k;
            src[r] = mat + col + k * ld;
        }
    }
    const bool full = wave < G::NI % G::NW || G::PMAX == G::PMIN;
    // The padded k of both operands are zero: the right one's are stored (H past D, d
    // past the tokens and words), the left one's are read from the header's zeros.
    // (With values of V in their place, a word of -inf made 0 times -inf, a NaN.)
    const int64_t lkmax = LOGITS ? a.D : (DV ? a.Tp : kmax);
    // elements from one step to the next
    const int64_t rstep = RK ? 32 : 32 * ldr, lstep = LK ? 32 : 32 * ldl;
    // `ends`: the step may reach past lkmax (its last two do)
    auto dma = [&](int u, int slot, bool ends) {
        // the second part of d: the same rows of H, columns of dS further on
        const bool second = PARTS == 2 && kb + u >= part;
        const int64_t su = kb + u - (second ? part : 0);
        const int64_t roff = su * rstep + (second ? a.lo : 0), loff = su * lstep;
        const bool past = ends && 32 * su + 32 > lkmax;
#pragma unroll
        for (int r = 0; r < G::PMAX; ++r) {
            if (r >= G::PMIN && !full) continue;
            const int v0 = wave + G::NW * r;
            const uint16_t *p = src[r] + (v0 < G::RU ? roff : loff);
            if (past && v0 >= G::RU && 32 * su + kof[r] >= lkmax)
                p = reinterpret_cast<const uint16_t *>(a.hdr + ZEROS);
            __builtin_amdgcn_global_load_lds(reinterpret_cast<const uint4 *>(p),
                                             reinterpret_cast<uint4 *>(s_mem + slot * G::SLOT + (v0 << 10)), 16, 0, 0);
        }
    };

    f32x4_t acc[MF][NF];
#pragma unroll
    for (int i = 0; i < MF; ++i)
#pragma unroll
        for (int j = 0; j < NF; ++j) acc[i][j] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};

    if (ku > 0) {
        for (int c = 0; c < G::NS && c < ku; ++c) dma(c, c, true);
        bf16x8_t rf[2][MF], lf[2][NF];
        auto frag_k = [&](int base) { return *reinterpret_cast<const bf16x8_t *>(s_mem + base); };
        // (k as row) the lane's bytes of even and of odd fragments
        const int tkey = 4 * (g & 1) + (r16 >> 2);
        const int tbase = (g >> 1) * 8192 + tkey * 64 + (r16 & 3) * 8;
        const int t0 = tbase + 32 * (g & 1), t1 = tbase + 32 * (1 - (g & 1));
        auto frag_tr = [&](int base, int f) {
            const uint8_t *p = s_mem + base + ((f & 1) ? t1 : t0) + (f >> 1) * 512;
            return read_tr(p, p + 4096);
        };
        const int lrow = LOGITS ? wn * NF * 16 + (r16 >> 2) * (4 * NF) + (r16 & 3) : 0;
        const int swz = (g ^ (-(r16 >> 2) & 3)) << 4;
        const int lbase = G::RU * 1024 + lrow * 64 + swz, rbase = (wm * MF * 16 + r16) * 64 + swz;
        auto read_l = [&](int p, int slot, int j) {
            const int sb = slot * G::SLOT;
            if constexpr (LK) lf[p][j] = frag_k(sb + lbase + j * 256);
            else lf[p][j] = frag_tr(sb + G::RU * 1024 + wn * NF * 256, j);
        };
        auto read_r = [&](int p, int slot, int i) {
            const int sb = slot * G::SLOT;
            if constexpr (RK) rf[p][i] = frag_k(sb + rbase + i * 1024);
            else rf[p][i] = frag_tr(sb + wm * MF * 256, i);
        };
        auto wait_steps = [&](auto n) {  // until at most n steps of DMAs are in flight
            constexpr int N = decltype(n)::value;
            if (full) wait_vm<N * G::PMAX>();
            else wait_vm<N * G::PMIN>();
        };
        if (ku >= G::NS) wait_steps(std::integral_constant<int, G::NS - 1>{});
        else wait_vm<0>();
        lds_barrier();
#pragma unroll
        for (int j = 0; j < NF; ++j) read_l(0, 0, j);
#pragma unroll
        for (int i = 0; i < MF; ++i) read_r(0, 0, i);
        int slot = 0;
        // step u: its fragments are in registers once the barrier's LDS wait is
        // over, for every wave, so its slot takes step u + NS. A row of products
        // at a time: the reads of step u + 1 go with the first rows, so that they
        // are over by the last, the DMAs with the last ones.
        constexpr int READS = MF + NF, HALF = MF > 1 ? MF / 2 : 1, PER = (READS + HALF - 1) / HALF;
        auto step = [&](int u, int p, auto inside) {
            // inside: neither this step's DMAs nor those before are the last
            constexpr bool IN = decltype(inside)::value;
            const bool more = IN || u + G::NS < ku;
            if (more) wait_steps(std::integral_constant<int, G::NS - 2>{});
            else wait_vm<0>();
            lds_barrier();
            const int next = (slot + 1 == G::NS) ? 0 : slot + 1;
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int i = 0; i < MF; ++i) {
#pragma unroll
                for (int q = 0; q < PER; ++q) {
                    const int k = i * PER + q;
                    if (i >= HALF || k >= READS) continue;
                    if (k < NF) read_l(1 - p, next, k);
                    else read_r(1 - p, next, k - NF);
                }
                if (i == MF - 1 - (MF > 1) && more) dma(u + G::NS, slot, !IN);
#pragma unroll
                for (int j = 0; j < NF; ++j)
                    acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(lf[p][j], rf[p][i], acc[i][j], 0, 0, 0);
                __builtin_amdgcn_sched_barrier(0);
            }
            slot = next;
        };
        int u = 0;
        for (; u + 1 + G::NS < ku - 2; u += 2) {
            step(u, 0, std::true_type{});
            step(u + 1, 1, std::true_type{});
        }
        for (; u < ku; u += 2) {
            step(u, 0, std::false_type{});
            step(u + 1, 1, std::false_type{});
        }
    }

    const int64_t rbeg = int64_t(by) * G::BR + 16 * (wm * MF) + r16;  // right row of group i: + 16 i
    if constexpr (EPI == EPI_STATS) {
        // per token: the largest of the tile's logits, the sum against it
        lds_barrier();
        float *s_max = reinterpret_cast<float *>(s_mem), *s_sum = s_max + WN * G::BR;
        const int64_t w0 = a.v0 + int64_t(bx) * G::BL + 16 * (wn * NF) + 4 * NF * g;
#pragma unroll
        for (int i = 0; i < MF; ++i) {
            const int64_t row = rbeg + 16 * i;
            const int tg = (row < a.Tp) ? a.tgt[row] : -1;
            float m = -__builtin_inff();
            bool nan = false;
#pragma unroll
            for (int j = 0; j < NF; ++j)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int64_t w = w0 + 4 * j + r;
                    if (w >= a.N) continue;
                    const float z = acc[i][j][r];
                    if (w == tg) a.ztgt[row] = z;
                    nan |= !(z == z);
                    m = z > m ? z : m;
                }
            float s = 0.0f;
            // against a finite value: a lane whose words are all -inf (or absent) adds 0
            const float ref = (m == -__builtin_inff()) ? 0.0f : m;
#pragma unroll
            for (int j = 0; j < NF; ++j)
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    if (w0 + 4 * j + r < a.N) s += __builtin_amdgcn_exp2f((acc[i][j][r] - ref) * LOG2E);
            if (nan) s = __builtin_nanf("");
            // join the four lanes of the token
#pragma unroll
            for (int d = 16; d < 64; d <<= 1) join_stats(m, s, __shfl_xor(m, d), __shfl_xor(s, d));
            if (g == 0) {
                s_max[wn * G::BR + 16 * (wm * MF + i) + r16] = m;
                s_sum[wn * G::BR + 16 * (wm * MF + i) + r16] = s;
            }
        }
        __syncthreads();
        for (int q = t; q < G::BR; q += 64 * G::NW) {
            float m = s_max[q], s = s_sum[q];
#pragma unroll
            for (int w = 1; w < WN; ++w) join_stats(m, s, s_max[w * G::BR + q], s_sum[w * G::BR + q]);
            const int64_t row = int64_t(by) * G::BR + q;
            if (row < live) a.stat[int64_t(bx) * a.Tp + row] = make_float2(m, s);
        }
    } else if constexpr (EPI == EPI_PROB) {
        // d = g (exp(z - lse) - onehot); 0 for padded tokens and words. bf16 results
        // take it rounded to bf16: at most 2^-9 of each value, which with the rounding
        // of the results makes the gradients' relative error 2.2e-3 to 2.5e-3 where that
        // rounding alone makes 1.7e-3, and a second part would double two of the three
        // products. A dV of 32 bits is asked for to be better than that: it takes what
        // remains as a second part (2^-18 is lost).
        const int64_t w0 = int64_t(bx) * G::BL + 16 * (wn * NF) + 4 * NF * g;
#pragma unroll
        for (int i = 0; i < MF; ++i) {
            const int64_t row = rbeg + 16 * i;
            const bool in = row < live;
            const int64_t tg = int64_t(a.tgt[row]) - a.v0;
            const float lse = a.lse[row] , gg = a.g[row];
            float v[4 * NF];
#pragma unroll
            for (int j = 0; j < NF; ++j)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int64_t w = w0 + 4 * j + r;
                    float p = __builtin_amdgcn_exp2f((acc[i][j][r] - lse) * LOG2E);
                    if (w == tg) p -= 1.0f;
                    v[4 * j + r] = (in && a.v0 + w < a.N) ? gg * p : 0.0f;
                }
            u32x4_t *q = reinterpret_cast<u32x4_t *>(a.dS + row * a.dsp + w0);
#pragma unroll
            for (int h = 0; h < NF / 2; ++h) {
                u32x4_t hi;
#pragma unroll
                for (int e = 0; e < 4; ++e) hi[e] = pack_bf16x2(v[8 * h + 2 * e], v[8 * h + 2 * e + 1]);
                q[h] = hi;
                if (a.lo == 0) continue;
                u32x4_t lo;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float x = v[8 * h + 2 * e] - __uint_as_float(hi[e] << 16);
                    const float y = v[8 * h + 2 * e + 1] - __uint_as_float(hi[e] & 0xffff0000u);
                    // (nothing remains of what is no number)
                    lo[e] = pack_bf16x2(x - x == 0.0f ? x : 0.0f, y - y == 0.0f ? y : 0.0f);
                }
                *reinterpret_cast<u32x4_t *>(a.dS + row * a.dsp + w0 + a.lo + 8 * h) = lo;
            }
        }
    } else if constexpr (EPI == EPI_DH) {
        // fp32 sums over the pieces, each split its own
        float *o = a.dHp + int64_t(z) * a.Tp * a.Dp;
        const int64_t c0 = int64_t(bx) * G::BL + 16 * (wn * NF) + 4 * g;
#pragma unroll
        for (int i = 0; i < MF; ++i) {
            const int64_t row = rbeg + 16 * i;
            if (row >= live) continue;
#pragma unroll
            for (int j = 0; j < NF; ++j) {
                const int64_t c = c0 + 16 * j;
                if (c >= a.D) continue;  // (D is a multiple of 8)
                f32x4_t *q = reinterpret_cast<f32x4_t *>(o + row * a.Dp + c);
                *q = a.first ? acc[i][j] : *q + acc[i][j];
            }
        }
    } else {
        const int64_t c0 = int64_t(bx) * G::BL + 16 * (wn * NF) + 4 * g;
#pragma unroll
        for (int i = 0; i < MF; ++i) {
            const int64_t w = a.v0 + rbeg + 16 * i;
            if (w >= a.N || rbeg + 16 * i >= a.vp) continue;
#pragma unroll
            for (int j = 0; j < NF; ++j) {
                const int64_t c = c0 + 16 * j;
                if (c >= a.D) continue;
                f32x4_t v = acc[i][j];
                if (a.dv_bf16) {
                    uint16_t *q = static_cast<uint16_t *>(a.dV) + w * a.lddv + c;
                    if (a.dv_vec) {
                        uint2 *q2 = reinterpret_cast<uint2 *>(q);
                        if (a.accumulate) {
                            const uint2 o = *q2;
                            v += f32x4_t{__uint_as_float(o.x << 16), __uint_as_float(o.x & 0xffff0000u),
                                         __uint_as_float(o.y << 16), __uint_as_float(o.y & 0xffff0000u)};
                        }
                        *q2 = make_uint2(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]));
                    } else {
#pragma unroll
                        for (int r = 0; r < 4; ++r)
                            q[r] = f32_to_bf16(a.accumulate ? bf16_to_f32(q[r]) + v[r] : v[r]);
                    }
                } else {
                    float *q = static_cast<float *>(a.dV) + w * a.lddv + c;
                    if (a.dv_vec) {
                        f32x4_t *q4 = reinterpret_cast<f32x4_t *>(q);
                        *q4 = a.accumulate ? *q4 + v : v;
                    } else {
#pragma unroll
                        for (int r = 0; r < 4; ++r) q[r] = a.accumulate ? q[r] + v[r] : v[r];
                    }
                }
            }
        }
    }
}

template <int EPI, int MF, int NF, int WM, int WN>
__global__ __launch_bounds__(64 * WM * WN) __attribute__((amdgpu_waves_per_eu(WM * WN / 4, WM * WN / 4)))
void xent_gemm(const XArgs a)
{
    xent_tile<EPI, MF, NF, WM, WN>(a, a.hdr[0]);
}

// The tiles by the tokens that have a loss, which only the GPU knows.
template <int EPI>
__global__ __launch_bounds__(512) __attribute__((amdgpu_waves_per_eu(2, 2))) void xent_gemm_live(const XArgs a)
{
    const int live = a.hdr[0];
    if (xent_half_tiles<EPI>(a, live)) xent_tile<EPI, 4, 4, 2, 4>(a, live);
    else xent_tile<EPI, 8, 4, 2, 4>(a, live);
}

// A token's tiles joined: TOK tokens a block, XT / TOK threads each over the
// tiles, their pairs then joined in order. (One block of 16 threads a token took
// 22 us for 594 tiles, with any number of tokens.)
template <int TOK>
__global__ __launch_bounds__(XT) void xent_join_kernel(const XArgs a, int tiles)
{
    constexpr int PARTS = XT / TOK;
    __shared__ float s_m[PARTS][TOK + 1], s_s[PARTS][TOK + 1];
    const int tok = threadIdx.x % TOK, part = threadIdx.x / TOK;
    const int64_t m = int64_t(blockIdx.x) * TOK + tok;
    const int row = m < a.T ? a.pos[m] : -1;
    float mx = -__builtin_inff(), s = 0.0f;
    if (row >= 0)
#pragma unroll 4
        for (int q = part; q < tiles; q += PARTS) {
            const float2 v = a.stat[int64_t(q) * a.Tp + row];
            join_stats(mx, s, v.x, v.y);
        }
    s_m[part][tok] = mx;
    s_s[part][tok] = s;
#pragma unroll
    for (int h = PARTS / 2; h > 0; h >>= 1) {
        __syncthreads();
        if (part < h) {
            join_stats(mx, s, s_m[part + h][tok], s_s[part + h][tok]);
            s_m[part][tok] = mx;
            s_s[part][tok] = s;
        }
    }
    if (part != 0 || m >= a.T) return;
    // (of the loss only the smaller terms are rounded: mx is often near z)
    a.lse_out[m] = row >= 0 ? mx + logf(s) : 0.0f;
    a.loss_out[m] = row >= 0 ? (mx - a.ztgt[row]) + logf(s) : 0.0f;
}

// dH rows from the sums (0 for tokens without a loss). One block per token.
__global__ __launch_bounds__(XT) void xent_dh_kernel(const XArgs a)
{
    const int64_t m = blockIdx.x;
    const int row = a.pos[m], live = a.hdr[0];
    const bool half = a.T <= 128 || (a.T <= HALF_TOKENS && xent_half_tiles<EPI_DH>(a, live));
    const int splits = half ? xent_tiles<EPI_DH, 128, 256>(a, live).splits : xent_tiles<EPI_DH, 256, 256>(a, live).splits;
    for (int64_t c = 4 * threadIdx.x; c < a.D; c += 4 * XT) {
        f32x4_t v = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
        if (row >= 0) {
            const float *q = a.dHp + int64_t(row) * a.Dp + c;
#pragma unroll 8
            for (int z = 0; z < splits; ++z) v += *reinterpret_cast<const f32x4_t *>(q + int64_t(z) * a.Tp * a.Dp);
        }
        uint16_t *o = a.dH + m * a.lddh + c;
        if (a.dh_vec) *reinterpret_cast<uint2 *>(o) = make_uint2(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]));
        else
#pragma unroll
            for (int r = 0; r < 4; ++r) o[r] = f32_to_bf16(v[r]);
    }
}

// ---------------------------------------------------------------------------
// Host side.
// ---------------------------------------------------------------------------
constexpr int64_t PIECE_BYTES = int64_t(256) << 20;  // of d

struct XLayout {
    int64_t Tp, Dp, tiles, vp, dsp;
    int hsplit;
    size_t rows, pos, tgt, lse, g, ztgt, hc, stat, ds, dhp, total;
};

XLayout xent_layout(bool grad, int64_t T, int64_t N, int64_t D)
{
    XLayout l{};
    l.Tp = std::max<int64_t>(1, (T + ROW_PAD - 1) / ROW_PAD) * ROW_PAD;
    l.Dp = (D + 63) / 64 * 64;
    l.tiles = (N + VBLK - 1) / VBLK;
    size_t at = 256;
    auto take = [&](size_t bytes) {
        const size_t p = at;
        at += align256(bytes);
        return p;
    };
    l.rows = take(size_t(l.Tp) * 4);
    l.pos = take(size_t(std::max<int64_t>(T, 1)) * 4);
    l.tgt = take(size_t(l.Tp) * 4);
    l.hc = take(size_t(l.Tp) * size_t(l.Dp) * 2);
    if (!grad) {
        l.ztgt = take(size_t(l.Tp) * 4);
        l.stat = take(size_t(l.tiles) * size_t(l.Tp) * 8);
    } else {
        l.lse = take(size_t(l.Tp) * 4);
        l.g = take(size_t(l.Tp) * 4);
        // words of a piece: as many as fit, in whole rounds of tiles over the 256
        // compute units where that leaves one round or more
        int64_t most = std::max<int64_t>(1, PIECE_BYTES / (l.Tp * 2 * VBLK));
        const int64_t rt = l.Tp / 256, round = 256 / std::gcd<int64_t>(256, rt);
        if (most >= round) most = most / round * round;
        l.vp = std::min(most, l.tiles) * VBLK;
        // room for two parts of d: of the whole vocabulary where that fits a piece's
        // space, of one tile of words at least
        l.dsp = std::max<int64_t>({l.vp, 2 * VBLK, std::min<int64_t>(2 * l.vp, most * VBLK)});
        l.ds = take(size_t(l.Tp) * size_t(l.dsp) * 2);
        // splits of dH's depth: until its launch fills the compute units
        const int64_t blocks = (l.Tp / 256) * ((D + 255) / 256);
        l.hsplit = int(std::clamp<int64_t>(256 / blocks, 1, std::max<int64_t>(1, std::min<int64_t>(l.vp / 512, 32))));
        l.dhp = take(size_t(l.hsplit) * size_t(l.Tp) * size_t(l.Dp) * 4);
    }
    l.total = at;
    return l;
}

// KERNEL takes tiles of BR x BL at least.
template <auto KERNEL, int BR, int BL, int THREADS, size_t LDS>
hipError_t launch_gemm_tiles(const XArgs &a, int64_t right, int64_t left, int splits, hipStream_t st)
{
    static std::atomic<bool> lds_set{false};  // the ring exceeds the default dynamic LDS limit
    if (!lds_set.load(std::memory_order_relaxed)) {
        const hipError_t e =
            hipFuncSetAttribute(reinterpret_cast<const void *>(KERNEL), hipFuncAttributeMaxDynamicSharedMemorySize, int(LDS));
        if (e != hipSuccess) return e;
        lds_set.store(true, std::memory_order_relaxed);
    }
    const int64_t blocks = (right + BR - 1) / BR * ((left + BL - 1) / BL) * splits;
    if (blocks == 0) return hipSuccess;
    hipLaunchKernelGGL(KERNEL, dim3(unsigned(blocks)), dim3(THREADS), LDS, st, a);
    return hipGetLastError();
}

template <int EPI, int MF, int NF, int WM, int WN>
hipError_t launch_gemm_shape(const XArgs &a, int64_t right, int64_t left, int splits, hipStream_t st)
{
    using G = XShape<MF, NF, WM, WN>;
    return launch_gemm_tiles<&xent_gemm<EPI, MF, NF, WM, WN>, G::BR, G::BL, 64 * G::NW, G::LDS>(a, right, left, splits, st);
}

// Token tiles by the number of tokens. d's rows are read 64 deep by dV, so its
// tiles have 64 or more.
template <int EPI>
hipError_t launch_tokens(const XArgs &a, int64_t left, int splits, hipStream_t st)
{
    if constexpr (EPI == EPI_STATS) {
        if (a.T <= 16) return launch_gemm_shape<EPI, 1, 4, 1, 4>(a, a.T, left, splits, st);
        if (a.T <= 32) return launch_gemm_shape<EPI, 1, 4, 2, 4>(a, a.T, left, splits, st);
    }
    if (a.T <= 64) return launch_gemm_shape<EPI, 2, 4, 2, 4>(a, a.T, left, splits, st);
    if (a.T <= 128) return launch_gemm_shape<EPI, 4, 4, 2, 4>(a, a.T, left, splits, st);
    using H = XShape<4, 4, 2, 4>;
    using W = XShape<8, 4, 2, 4>;
    if (a.T <= HALF_TOKENS)
        return launch_gemm_tiles<&xent_gemm_live<EPI>, H::BR, H::BL, 512, (W::LDS > H::LDS ? W::LDS : H::LDS)>(a, a.T, left, splits, st);
    return launch_gemm_shape<EPI, 8, 4, 2, 4>(a, a.T, left, splits, st);
}

XArgs xent_args(const XentCall &c, const XLayout &l)
{
    char *ws = static_cast<char *>(c.ws);
    XArgs a{};
    a.hdr = reinterpret_cast<int32_t *>(ws);
    a.rows = reinterpret_cast<int32_t *>(ws + l.rows);
    a.pos = reinterpret_cast<int32_t *>(ws + l.pos);
    a.tgt = reinterpret_cast<int32_t *>(ws + l.tgt);
    a.Hc = reinterpret_cast<uint16_t *>(ws + l.hc);
    a.H = static_cast<const uint16_t *>(c.H);
    a.V = static_cast<const uint16_t *>(c.V);
    a.ldh = c.ldh;
    a.ldv = c.ldv;
    a.T = c.T;
    a.N = c.N;
    a.D = c.D;
    a.Tp = l.Tp;
    a.Dp = l.Dp;
    a.target = c.target;
    a.err = c.err;
    return a;
}

// `rows`: the compact rows that the call's tiles read (a multiple of 16)
hipError_t launch_rows(const XArgs &a, int64_t rows, hipStream_t st)
{
    const dim3 grid(unsigned(rows / (XR / XT)));
    if (a.T <= ROWS_ONE) {
        hipLaunchKernelGGL((xent_pack_kernel<true>), grid, dim3(XR), 0, st, a);
        return hipGetLastError();
    }
    hipLaunchKernelGGL(xent_rows_kernel, dim3(1), dim3(XR), 0, st, a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((xent_pack_kernel<false>), grid, dim3(XR), 0, st, a);
    return hipGetLastError();
}

}  // namespace

size_t xent_ws_bytes(bool grad, int64_t T, int64_t N, int64_t D) { return xent_layout(grad, T, N, D).total; }

hipError_t launch_xent_loss(const XentCall &c, hipStream_t st)
{
    const XLayout l = xent_layout(false, c.T, c.N, c.D);
    XArgs a = xent_args(c, l);
    a.ztgt = reinterpret_cast<float *>(static_cast<char *>(c.ws) + l.ztgt);
    a.stat = reinterpret_cast<float2 *>(static_cast<char *>(c.ws) + l.stat);
    a.loss_out = c.loss;
    a.lse_out = c.lse;
    hipError_t e = launch_rows(a, c.T <= 16 ? 16 : (c.T <= 32 ? 32 : a.Tp), st);
    if (e != hipSuccess) return e;
    // A launch holds fewer than 2^32 work items, 512 or fewer of a tile: the tiles
    // of larger vocabularies go over several.
    const int64_t rt = c.T <= 128 ? 1 : (c.T <= HALF_TOKENS ? (c.T + 127) / 128 : (c.T + 255) / 256);
    const int64_t most = ((int64_t(1) << 32) - 1) / (512 * rt);
    float2 *const stat = a.stat;
    for (int64_t t0 = 0; t0 < l.tiles; t0 += most) {
        a.v0 = t0 * VBLK;
        a.vp = std::min(most, l.tiles - t0) * VBLK;
        a.stat = stat + t0 * a.Tp;
        if ((e = launch_tokens<EPI_STATS>(a, a.vp, 1, st)) != hipSuccess) return e;
    }
    a.stat = stat;
    // few tokens: a block each; else eight, whose pairs lie next to each other
    if (c.T < 512) hipLaunchKernelGGL((xent_join_kernel<1>), dim3(unsigned(c.T)), dim3(XT), 0, st, a, int(l.tiles));
    else hipLaunchKernelGGL((xent_join_kernel<8>), dim3(unsigned((c.T + 7) / 8)), dim3(XT), 0, st, a, int(l.tiles));
    return hipGetLastError();
}

hipError_t launch_xent_grad(const XentCall &c, hipStream_t st)
{
    const XLayout l = xent_layout(true, c.T, c.N, c.D);
    XArgs a = xent_args(c, l);
    char *ws = static_cast<char *>(c.ws);
    a.lse_in = c.lse_in;
    a.g_in = c.g;
    a.lse = reinterpret_cast<float *>(ws + l.lse);
    a.g = reinterpret_cast<float *>(ws + l.g);
    a.dS = reinterpret_cast<uint16_t *>(ws + l.ds);
    a.dsp = l.dsp;
    a.dHp = reinterpret_cast<float *>(ws + l.dhp);
    a.hsplit = l.hsplit;
    a.dH = static_cast<uint16_t *>(c.dH);
    a.lddh = c.lddh;
    a.dh_vec = (reinterpret_cast<uintptr_t>(c.dH) | uintptr_t(2 * c.lddh)) % 8 == 0;
    a.dV = c.dV;
    a.lddv = c.lddv;
    a.dv_bf16 = c.dv_dtype == BSQ_BF16;
    const int64_t vb = a.dv_bf16 ? 8 : 16;
    a.dv_vec = (reinterpret_cast<uintptr_t>(c.dV) | uintptr_t(vb / 4 * c.lddv)) % vb == 0;
    a.accumulate = c.accumulate;
    // two parts of d for a dV of 32 bits: half the words a piece, in the same space
    const bool two = c.dV && !a.dv_bf16;
    const int64_t vp = two ? l.dsp / 2 / VBLK * VBLK : l.vp;
    a.lo = two ? vp : 0;
    hipError_t e = launch_rows(a, a.Tp, st);
    for (int64_t v0 = 0; e == hipSuccess && v0 < c.N; v0 += vp) {
        a.v0 = v0;
        a.vp = std::min(vp, (c.N - v0 + VBLK - 1) / VBLK * VBLK);
        a.first = v0 == 0;
        if ((e = launch_tokens<EPI_PROB>(a, a.vp, 1, st)) != hipSuccess) break;
        if ((e = launch_tokens<EPI_DH>(a, c.D, l.hsplit, st)) != hipSuccess) break;
        if (two) e = launch_gemm_shape<EPI_DV2, 8, 4, 2, 4>(a, a.vp, c.D, 1, st);
        else if (c.dV) e = launch_gemm_shape<EPI_DV, 8, 4, 2, 4>(a, a.vp, c.D, 1, st);
    }
    if (e != hipSuccess || c.T == 0) return e;
    hipLaunchKernelGGL(xent_dh_kernel, dim3(unsigned(c.T)), dim3(XT), 0, st, a);
    return hipGetLastError();
}

}  // namespace bsq
