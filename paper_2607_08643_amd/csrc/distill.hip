// Distillation of a student, given by hidden states H [T][D] and head weights V [N][D],
// from a teacher's top logits a [T][K] of the words ids [T][K], at a scale s (one over the
// temperature), and its gradient:
//   p_k = exp(s a_k - norm)  (norm: the log of the sum over the teacher's whole vocabulary,
//                             or over the K words),  P = sum p_k,
//   q = softmax(s H V^T),  loss = sum_k p_k (log p_k - log q_id_k),
//   d = g s (P q - sum of p_k at its word),  dH = d V,  dV = d^T H.
//
// The products are those of the cross entropy (vocab_product.h). What a token has of its
// teacher is K words: they are sorted by word once, with the place where each 256-word
// tile's begin, so that a tile finds the few of its own (64 of 151936 words: one in
// ten tiles) while it holds the logits in registers. The loss is joined from the tiles'
// statistics and these logits in 64 bits.
//
// What is kept: the loss can leave the exponentials of its logits, 16 bits each, and what
// it found of tokens and teacher for the gradient, which then makes d in one pass over
// memory and has one product less to do: 6 bytes a logit moved against 2 D operations. (d
// is rounded to bf16 all the same, by up to 2^-8, beside which 2^-11 adds nothing to speak
// of; for a dV of 32 bits the logits are made again.)
//
// Bound by the matrix cores from some hundred tokens on: 4096 tokens of 151936 words, 4096
// inputs: logits with what is kept of them 4.55 ms (1.12 PFLOP/s), d 0.44 (5.6 TB/s), dH 4.0
// (1.27), dV 4.5 (1.14), as a profiler sees them (the step 4% longer than without); the
// teacher's words 18 to 21 us. 37 tokens of 32003 words, 1000 inputs:
// the logits 18 to 19 us (one reading of V, 3.4 to 3.6 TB/s), three short launches 14.
#include "vocab_product.h"
#include "vocab_rows.h"

namespace bsq {
namespace {

constexpr int KMAX = BSQ_MAX_TOP;
static_assert(KMAX <= XT, "a thread for every word of a token");

struct TeacherArgs {
    const int32_t *ids;
    const float *top, *norm;
    int64_t N, tiles;
    int K;
    float scale;
    int64_t *live;    // [T]: 0, or -1 for a token without a loss
    int32_t *sid;     // [T][K]
    float *sp;        // [T][K]
    uint16_t *off;    // [T][tiles + 1]
    float *total;     // [T]: sum of p
    double *self;     // [T]: sum of p log p
    int32_t *err;
};

__device__ __forceinline__ double block_sum64(double v, double *s)
{
    const int t = threadIdx.x;
    v = wave_sum(v);
    __syncthreads();
    if ((t & 63) == 0) s[t >> 6] = v;
    __syncthreads();
    v = 0.0;
    for (int w = 0; w < XT / 64; ++w) v += s[w];
    return v;
}

// A token's words in order, their probabilities, and each tile's first. One block a token.
__global__ __launch_bounds__(XT) void distill_teacher_kernel(const TeacherArgs a)
{
    __shared__ uint64_t s_key[KMAX];
    __shared__ int32_t s_id[KMAX];
    __shared__ double s_sum[XT / 64], s_max[XT / 64];
    const int t = threadIdx.x;
    const int64_t m = blockIdx.x;
    int32_t id = -1;
    double x = -__builtin_inf();  // (its product with the scale is not rounded)
    if (t < a.K) {
        id = a.ids[m * a.K + t];
        if (id >= a.N) {
            if (a.err) atomicOr(a.err, BSQ_DEVERR_BAD_SET);
            id = -1;
        }
        x = double(a.top[m * a.K + t]) * double(a.scale);
        // (a word of -inf is not there: its probability is 0)
        if (id < 0 || x == -__builtin_inf()) {
            id = -1;
            x = -__builtin_inf();
        }
    }
    const bool there = id >= 0;
    // absent words last, each key another
    const uint64_t key = (uint64_t(uint32_t(there ? id : INT32_MAX)) << 16) | uint32_t(t);
    s_key[t] = key;
    // The largest in 64 bits, so that its exponential is 1: rounded to 32 it is some 2^-24 of
    // itself off, which leaves exp's range from products of 10^10 on. (A NaN counts as nothing.)
    double mx = lane_value(wave_scan(x, -__builtin_inf(), [](double a, double b) { return fmax(a, b); }), 63);
    if ((t & 63) == 0) s_max[t >> 6] = mx;
    const bool live = __syncthreads_or(there);
    for (int w = 0; w < XT / 64; ++w) mx = fmax(mx, s_max[w]);
    double logp, p;
    if (a.norm) {
        logp = x - double(a.norm[m]);
    } else {
        const double sum = block_sum64(there ? exp(x - mx) : 0.0, s_sum);
        logp = (x - mx) - log(sum);
    }
    p = there ? exp(logp) : 0.0;
    const double total = block_sum64(p, s_sum);
    const double self = block_sum64(there && p != 0.0 ? p * logp : 0.0, s_sum);
    if (t < a.K) {
        int place = 0;
        for (int k = 0; k < a.K; ++k) place += s_key[k] < key ? 1 : 0;
        s_id[place] = there ? id : INT32_MAX;
        a.sid[m * a.K + place] = there ? id : INT32_MAX;
        a.sp[m * a.K + place] = float(p);
    }
    if (t == 0) {
        a.live[m] = live ? 0 : -1;
        a.total[m] = float(total);
        a.self[m] = self;
    }
    __syncthreads();
    for (int64_t tile = t; tile <= a.tiles; tile += XT) {
        const int64_t first = tile * VBLK;
        int lo = 0, hi = a.K;  // words below `first`
        while (lo < hi) {
            const int mid = (lo + hi) >> 1;
            if (s_id[mid] < first && s_id[mid] != INT32_MAX) lo = mid + 1;
            else hi = mid;
        }
        a.off[m * (a.tiles + 1) + tile] = uint16_t(lo);
    }
}

// A token's tiles joined, and its loss: TOK tokens a block, XT / TOK threads each over the
// tiles and the teacher's words, joined in order.
template <int TOK>
__global__ __launch_bounds__(XT) void distill_join_kernel(const XArgs a, const double *self, int tiles)
{
    constexpr int PARTS = XT / TOK;
    __shared__ float s_m[PARTS][TOK + 1], s_s[PARTS][TOK + 1];
    __shared__ double s_z[PARTS][TOK + 1];
    const int tok = threadIdx.x % TOK, part = threadIdx.x / TOK;
    const int64_t m = int64_t(blockIdx.x) * TOK + tok;
    const int row = m < a.T ? a.pos[m] : -1;
    float mx = -__builtin_inff(), s = 0.0f;
    double z = 0.0;
    if (row >= 0) {
#pragma unroll 4
        for (int q = part; q < tiles; q += PARTS) {
            const float2 v = a.stat[int64_t(q) * a.Tp + row];
            join_stats(mx, s, v.x, v.y);
        }
        for (int k = part; k < a.K; k += PARTS) {
            const float p = a.sp[m * a.K + k];
            if (p != 0.0f) z += double(p) * double(a.zk[m * a.K + k]);
        }
    }
    s_m[part][tok] = mx;
    s_s[part][tok] = s;
    s_z[part][tok] = z;
#pragma unroll
    for (int h = PARTS / 2; h > 0; h >>= 1) {
        __syncthreads();
        if (part < h) {
            join_stats(mx, s, s_m[part + h][tok], s_s[part + h][tok]);
            z += s_z[part + h][tok];
            s_m[part][tok] = mx;
            s_s[part][tok] = s;
            s_z[part][tok] = z;
        }
    }
    if (part != 0 || m >= a.T) return;
    const double lse = double(mx) + log(double(s));
    a.lse_out[m] = row >= 0 ? float(lse) : 0.0f;
    a.loss_out[m] = row >= 0 ? float(self[m] - z + double(a.total[m]) * lse) : 0.0f;
}

// d of a piece of the vocabulary from what the loss kept: a block has KV runs of eight words
// a thread of a row, all in flight at once (4096 tokens of 32768 words: 95 us, 5.7 TB/s;
// with one run a fifth more). The teacher's words, where P q and p may nearly cancel, are made
// from their logits in 32 bits and written over, a thread each.
constexpr int KV = 4;

__global__ __launch_bounds__(XT) void distill_kept_kernel(const XArgs a, int blocks)
{
    __shared__ int32_t s_id[KMAX];
    __shared__ float s_p[KMAX];
    const int t = threadIdx.x, live = a.hdr[0];
    const int64_t row = blockIdx.x / blocks;
    if (row >= (int64_t(live) + 63) / 64 * 64) return;  // (d's rows are read 64 deep by dV)
    const int64_t first = int64_t(blockIdx.x - row * blocks) * (8 * XT * KV), w0 = first + 8 * t;
    uint16_t *dS = a.dS + row * a.dsp;
    if (row >= live) {
#pragma unroll
        for (int j = 0; j < KV; ++j) {
            if (w0 + 8 * XT * j >= a.vp) break;
            *reinterpret_cast<u32x4_t *>(dS + w0 + 8 * XT * j) = u32x4_t{0u, 0u, 0u, 0u};
            if (a.lo) *reinterpret_cast<u32x4_t *>(dS + w0 + 8 * XT * j + a.lo) = u32x4_t{0u, 0u, 0u, 0u};
        }
        return;
    }
    u32x4_t code[KV];
    float f[KV];
#pragma unroll
    for (int j = 0; j < KV; ++j) {
        const int64_t w = w0 + 8 * XT * j, word = a.v0 + (w < a.vp ? w : 0);
        code[j] = *reinterpret_cast<const u32x4_t *>(a.kept + row * a.ldk + word);
        f[j] = a.kept_max[row * (a.ldk / 64) + word / 64];
    }
    const int64_t tok = a.rows[row], end_w = first + 8 * XT * KV < a.vp ? first + 8 * XT * KV : a.vp;
    const float lse = a.lse_in[tok], gg = a.g_in[tok] * a.scale, total = a.total[tok];
    // the teacher's words of the block, one a thread (v0, first and vp are whole tiles)
    const uint16_t *off = a.off + tok * (a.tiles + 1) + a.v0 / VBLK;
    const int beg = off[first / VBLK], count = off[end_w / VBLK] - beg;
    const int64_t at = tok * a.K + beg + t;
    int32_t id = -1;
    float p = 0.0f, z = 0.0f;
    if (t < count) {
        id = a.sid[at];
        p = a.sp[at];
        z = a.zk[at];
        s_id[t] = id;
        s_p[t] = p;
    }
#pragma unroll
    for (int j = 0; j < KV; ++j) {
        const int64_t w = w0 + 8 * XT * j, word = a.v0 + w;
        if (w >= a.vp) break;
        // (a group of -inf is 0, but for a row without a softmax: lse is NaN, or -inf itself)
        const float q = f[j] == -__builtin_inff() && lse > -__builtin_inff() ? 0.0f : gg * (__builtin_amdgcn_exp2f((f[j] - lse) * LOG2E) * total);
        float v[8];
#pragma unroll
        for (int k = 0; k < 8; ++k)
            v[k] = word + k < a.N ? q * kept_value((k & 1) ? code[j][k >> 1] >> 16 : code[j][k >> 1] & 0xffffu) : 0.0f;
        put_d(dS + w, v, a.lo);
    }
    __syncthreads();  // (the words above are written before those of the teacher)
    if (t >= count || (t > 0 && s_id[t - 1] == id)) return;
    float d = gg * (__builtin_amdgcn_exp2f((z - lse) * LOG2E) * total) - gg * p;
    for (int k = t + 1; k < count && s_id[k] == id; ++k) d -= gg * s_p[k];  // (a word listed again)
    uint16_t *out = dS + (id - a.v0);
    const uint32_t hi = pack_bf16x2(d, 0.0f);
    out[0] = uint16_t(hi);
    if (a.lo) {
        const float x = d - __uint_as_float(hi << 16);
        out[a.lo] = uint16_t(pack_bf16x2(x - x == 0.0f ? x : 0.0f, 0.0f));
    }
}

// ---------------------------------------------------------------------------
// Host side.
// ---------------------------------------------------------------------------
// What the products need of tokens and teacher: compact rows, then a token's words and
// their tiles. It lies in the workspace, or first in what a loss keeps for its gradient.
struct SLayout {
    XLayout x;
    size_t live, sid, sp, off, total, zk, base_bytes;
    size_t codes, maxima, kept_bytes;   // kept: after the base
    size_t self, stat, ws_bytes;
    int narrow;
};

SLayout distill_layout(bool grad, int64_t T, int64_t N, int64_t D, int K)
{
    SLayout l{};
    l.x = xent_layout(grad, T, N, D);
    size_t at = align256(l.x.compact);
    auto take = [&](size_t bytes) {
        const size_t p = at;
        at += align256(bytes);
        return p;
    };
    const size_t t = size_t(std::max<int64_t>(T, 1));
    l.live = take(t * 8);
    l.sid = take(t * K * 4);
    l.sp = take(t * K * 4);
    l.off = take(t * size_t(l.x.tiles + 1) * 2);
    l.total = take(t * 4);
    l.zk = take(t * K * 4);
    l.base_bytes = at;
    l.codes = take(size_t(T) * size_t(l.x.tiles) * VBLK * 2);
    l.maxima = take(size_t(T) * size_t(l.x.tiles) * (VBLK / 64) * 4);
    l.kept_bytes = at;
    // workspace: the cross entropy's (its first part is the compact rows), the rest of the base
    at = align256(l.x.total) + (l.base_bytes - align256(l.x.compact));
    l.self = take(t * 8);
    // tiles of 128 words where 256 leave compute units idle (37 tokens of 32003 words, 1000
    // inputs: the loss's product 25 us with 126 tiles, 19 with 251)
    l.narrow = !grad && T <= 128 && l.x.tiles < 256;
    l.stat = l.narrow ? take(size_t(2 * l.x.tiles) * size_t(l.x.Tp) * 8) : l.x.stat;
    l.ws_bytes = at;
    return l;
}

// The arguments of the products and, `make`, the teacher's words.
hipError_t launch_teacher(const DistillCall &c, const SLayout &l, bool make, XArgs &a, hipStream_t st)
{
    char *ws = static_cast<char *>(c.x.ws);
    // (in the workspace the rest of the base follows the cross entropy's part)
    char *base = c.kept ? static_cast<char *>(c.kept) : ws;
    char *words = c.kept ? base : ws + (align256(l.x.total) - align256(l.x.compact));
    TeacherArgs h{};
    h.ids = c.ids;
    h.top = c.top;
    h.norm = c.norm;
    h.N = c.x.N;
    h.tiles = l.x.tiles;
    h.K = c.K;
    h.scale = c.scale;
    h.live = reinterpret_cast<int64_t *>(words + l.live);
    h.sid = reinterpret_cast<int32_t *>(words + l.sid);
    h.sp = reinterpret_cast<float *>(words + l.sp);
    h.off = reinterpret_cast<uint16_t *>(words + l.off);
    h.total = reinterpret_cast<float *>(words + l.total);
    h.self = reinterpret_cast<double *>(ws + l.self);
    h.err = c.x.err;
    XentCall x = c.x;
    x.target = h.live;
    x.err = nullptr;
    a = xent_args(x, l.x, base);
    a.sid = h.sid;
    a.sp = h.sp;
    a.off = h.off;
    a.total = h.total;
    a.zk = reinterpret_cast<float *>(words + l.zk);
    a.kept = c.kept ? reinterpret_cast<uint16_t *>(base + l.codes) : nullptr;
    a.kept_max = c.kept ? reinterpret_cast<float *>(base + l.maxima) : nullptr;
    a.ldk = l.x.tiles * VBLK;
    a.tiles = l.x.tiles;
    a.K = c.K;
    a.narrow = l.narrow;
    a.scale = c.scale;
    if (!make || c.x.T == 0) return hipSuccess;
    hipLaunchKernelGGL(distill_teacher_kernel, dim3(unsigned(c.x.T)), dim3(XT), 0, st, h);
    return hipGetLastError();
}

}  // namespace

size_t distill_ws_bytes(bool grad, int64_t T, int64_t N, int64_t D, int K) { return distill_layout(grad, T, N, D, K).ws_bytes; }

size_t distill_kept_bytes(int64_t T, int64_t N, int64_t D, int K) { return distill_layout(false, T, N, D, K).kept_bytes; }

hipError_t launch_distill_loss(const DistillCall &c, hipStream_t st)
{
    const SLayout l = distill_layout(false, c.x.T, c.x.N, c.x.D, c.K);
    XArgs a{};
    hipError_t e = launch_teacher(c, l, true, a, st);
    if (e != hipSuccess) return e;
    char *ws = static_cast<char *>(c.x.ws);
    a.stat = reinterpret_cast<float2 *>(ws + l.stat);
    a.loss_out = c.x.loss;
    a.lse_out = c.x.lse;
    if ((e = launch_stats<EPI_TSTATS>(a, l.x, st)) != hipSuccess) return e;
    const double *self = reinterpret_cast<const double *>(ws + l.self);
    const int tiles = int(l.x.tiles << l.narrow);
    if (a.T < 512) hipLaunchKernelGGL((distill_join_kernel<1>), dim3(unsigned(a.T)), dim3(XT), 0, st, a, self, tiles);
    else hipLaunchKernelGGL((distill_join_kernel<8>), dim3(unsigned((a.T + 7) / 8)), dim3(XT), 0, st, a, self, tiles);
    return hipGetLastError();
}

hipError_t launch_distill_grad(const DistillCall &call, hipStream_t st)
{
    // (nothing was kept of no tokens; 16 bits are too few for d in two parts)
    DistillCall c = call;
    if (c.x.T == 0 || (c.x.dV && c.x.dv_dtype == BSQ_F32)) c.kept = nullptr;
    const SLayout l = distill_layout(true, c.x.T, c.x.N, c.x.D, c.K);
    const bool kept = c.kept != nullptr;
    XArgs a{};
    const hipError_t e = launch_teacher(c, l, !kept, a, st);
    if (e != hipSuccess) return e;
    // (with what is kept nothing before the gradient's last launch looks at the ids)
    if (kept && c.x.err) {
        a.given = c.ids;
        a.err = c.x.err;
    }
    auto make_d = [&](const XArgs &piece) {
        if (!kept) return launch_tokens<EPI_TPROB>(piece, piece.vp, 1, st);
        const int64_t blocks = (piece.vp + 8 * XT * KV - 1) / (8 * XT * KV), rows = (piece.T + 63) / 64 * 64;
        if (rows == 0) return hipSuccess;
        hipLaunchKernelGGL(distill_kept_kernel, dim3(unsigned(rows * blocks)), dim3(XT), 0, st, piece, int(blocks));
        return hipGetLastError();
    };
    // Where tokens are few the rounding of d to bf16 does not average out over them, and the
    // products read and write the head either way: they take d in two parts.
    return c.x.T <= FEW_TOKENS ? launch_grad<true>(c.x, l.x, a, kept, st, make_d) : launch_grad<false>(c.x, l.x, a, kept, st, make_d);
}

}  // namespace bsq
