// Verification of drafted tokens against the target's probabilities, from given
// random numbers. Of a sequence with n drafted tokens x_i, target logits p_0 .. p_n and
// draft logits q_0 .. q_(n-1) (rows of a vocabulary), softmax at the sequence's
// temperature:
//   x_i is accepted while  u_i q_i(x_i) < p_i(x_i);
//   the token after the accepted ones is drawn from max(p_i - q_i, 0) where x_i was
//   refused, from p_n where none was: the first word whose cumulative sum exceeds r
//   times the whole.
// Without draft logits the drafts are certain: q_i(x_i) = 1, and x_i is taken out of p_i.
//
// Three launches: the largest logit and the sum of exponentials of every piece of
// every row that is needed; the pieces' sums of max(p - q, 0) of the one row where a
// draft was refused (every block first decides its sequence from the first launch's
// results); the draw, one block a sequence. No atomics but an OR of error bits: a result
// depends on the inputs alone.
//
// Sums and exponentials are 64-bit: a cumulative sum over 151936 words passes a given
// random number at the same word as the definition's only if the sum is off by much
// less than one word's share, and with exponentials of 32 bits one draw in some 200
// would be another word. The rows are read once from memory and, of one or two rows a
// sequence, once again from the caches.
#include <algorithm>

#include "vocab_rows.h"

namespace bsq {
namespace {

constexpr int DT = 256;                // threads of a block
constexpr int64_t VSTEP = 8 * DT;      // words of a vector a thread
constexpr int64_t MAX_PIECES = 64;     // of a row: one a lane
constexpr int MAXL = BSQ_MAX_DRAFTS;
constexpr double LOG2E_64 = 1.4426950408889634074;
static_assert(MAXL <= 64, "a lane for every drafted token");

enum { DRAW_TARGET, DRAW_REST, DRAW_OTHERS, DRAW_LARGEST, DRAW_NONE };

struct Piece {
    double sum;   // of exponentials against `top` (greedy rows: 0, or NaN where a logit is)
    float top;
    int32_t arg;  // greedy rows: lowest index of the largest
};

// What a sequence's drafts came to: `kind` of draw, the rows' largest logits and sums.
struct Decision {
    int32_t count, kind;
    float mp, mq;
    double sp, sq;
    int32_t token, arg;  // the refused token, the largest's index
    int32_t bits, pad;   // of the error word
};

struct DArgs {
    const void *P, *Q;
    int64_t B, N, pseq, prow, qseq, qrow;
    int L, rows, pieces;  // rows: of a sequence, L + 1 (+ L with draft logits)
    int64_t len;          // words of a piece
    const int32_t *tokens, *lens;
    const float *u, *r, *temp;
    int32_t *count, *out, *err;
    Piece *part;          // [B][rows][pieces]
    double *rest;         // [B][pieces]
    Decision *dec;        // [B]
};

// Drafted tokens of a sequence; a length outside 0 .. L is reported and clamped.
__device__ __forceinline__ int seq_len(const DArgs &a, int64_t b, bool &bad)
{
    if (!a.lens) return a.L;
    const int n = a.lens[b];
    if (n < 0 || n > a.L) bad = true;
    return n < 0 ? 0 : (n > a.L ? a.L : n);
}

// log2(e) over the temperature; 0 for a greedy sequence. (A temperature that is negative
// or not finite is reported and counts as 0.)
__device__ __forceinline__ double seq_scale(const DArgs &a, int64_t b, bool &bad)
{
    if (!a.temp) return LOG2E_64;
    const float t = a.temp[b];
    if (!(t >= 0.0f) || t == __builtin_inff()) {
        bad = true;
        return 0.0;
    }
    return t == 0.0f ? 0.0 : LOG2E_64 / double(t);
}

template <bool PB, bool QB>
struct Rows {
    const void *p, *q;
    __device__ __forceinline__ Rows(const DArgs &a, int64_t b, int64_t i)
    {
        const int64_t po = b * a.pseq + i * a.prow, qo = b * a.qseq + i * a.qrow;
        p = PB ? static_cast<const void *>(static_cast<const uint16_t *>(a.P) + po) : static_cast<const float *>(a.P) + po;
        q = QB ? static_cast<const void *>(static_cast<const uint16_t *>(a.Q) + qo) : static_cast<const float *>(a.Q) + qo;
    }
};

__device__ __forceinline__ float finite_ref(float m) { return m == -__builtin_inff() ? 0.0f : m; }

// Two pieces' largest logit and sum joined.
__device__ __forceinline__ void join(float &m, double &s, float m2, double s2, double c)
{
    const float mm = m2 > m ? m2 : m;
    const double ref = finite_ref(mm);
    s = s * exp2_64((m - ref) * c) + s2 * exp2_64((m2 - ref) * c);
    m = mm;
}

// The larger of two, of equal ones the lower index.
__device__ __forceinline__ void larger(float &m, int &arg, float m2, int arg2)
{
    if (m2 > m || (m2 == m && arg2 < arg)) {
        m = m2;
        arg = arg2;
    }
}

constexpr int NV = 4;  // vectors a thread reads together

template <bool BF16>
__device__ __forceinline__ void piece_stats(const void *row, int64_t n0, int64_t n1, double c, float &m, double &s, int &arg)
{
    m = -__builtin_inff();
    s = 0.0;
    arg = INT32_MAX;
    for (int64_t base = n0 + 8 * threadIdx.x; base < n1; base += NV * VSTEP) {
        Words8<BF16> w[NV];
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const int64_t at = base + k * VSTEP;
            w[k].load(row, at < n1 ? at : n1, n1);
        }
        if (c == 0.0) {
#pragma unroll
            for (int k = 0; k < NV; ++k)
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float z = w[k][e];
                    if (z > m) {
                        m = z;
                        arg = int(base + k * VSTEP + e);
                    }
                    if (!(z == z)) s = __builtin_nan("");
                }
            continue;
        }
        float mx = m;
#pragma unroll
        for (int k = 0; k < NV; ++k)
#pragma unroll
            for (int e = 0; e < 8; ++e) mx = fmaxf(mx, w[k][e]);
        const double ref = finite_ref(mx);
        if (mx > m) {
            s *= exp2_64((m - ref) * c);
            m = mx;
        }
#pragma unroll
        for (int k = 0; k < NV; ++k)
#pragma unroll
            for (int e = 0; e < 8; ++e) s += exp2_64((w[k][e] - ref) * c);
    }
}

// Largest logit and sum of every piece of every row that the sequence needs.
template <bool PB, bool QB>
__global__ __launch_bounds__(DT) void draft_rows_kernel(const DArgs a)
{
    __shared__ float s_m[DT / 64];
    __shared__ double s_s[DT / 64];
    __shared__ int s_arg[DT / 64];
    const int t = threadIdx.x, lane = t & 63, w = t >> 6;
    const int64_t items = a.B * a.rows * a.pieces;
    for (int64_t item = blockIdx.x; item < items; item += gridDim.x) {
        const int64_t rr = item / a.pieces, piece = item - rr * a.pieces, b = rr / a.rows;
        const int j = int(rr - b * a.rows);
        bool bad = false;
        const int n = seq_len(a, b, bad);
        const double c = seq_scale(a, b, bad);
        const bool target = j <= a.L;
        const int i = target ? j : j - a.L - 1;
        if (target ? i > n : (i >= n || c == 0.0)) continue;
        const Rows<PB, QB> rows(a, b, i);
        const int64_t n0 = piece * a.len, n1 = n0 + a.len < a.N ? n0 + a.len : a.N;
        float m;
        double s;
        int arg;
        if (target) piece_stats<PB>(rows.p, n0, n1, c, m, s, arg);
        else piece_stats<QB>(rows.q, n0, n1, c, m, s, arg);
        float wm = m;
        for (int d = 32; d > 0; d >>= 1) {
            const float m2 = __shfl_xor(wm, d);
            const int arg2 = __shfl_xor(arg, d);
            larger(wm, arg, m2, arg2);
        }
        if (c != 0.0) s *= exp2_64((m - double(finite_ref(wm))) * c);
        for (int d = 32; d > 0; d >>= 1) s += __shfl_xor(s, d);
        if (lane == 0) {
            s_m[w] = wm;
            s_s[w] = s;
            s_arg[w] = arg;
        }
        __syncthreads();
        if (t == 0) {
            for (int k = 1; k < DT / 64; ++k) {
                if (c != 0.0) {
                    join(wm, s, s_m[k], s_s[k], c);
                } else {
                    larger(wm, arg, s_m[k], s_arg[k]);
                    s += s_s[k];
                }
            }
            a.part[item] = Piece{s, wm, arg};
        }
        __syncthreads();
    }
}

// A row's pieces joined by a wave (every lane gets the result).
__device__ __forceinline__ void row_stats(const DArgs &a, int64_t b, int j, double c, float &m, double &s, int &arg)
{
    const int lane = threadIdx.x & 63;
    const bool in = lane < a.pieces;
    const Piece p = in ? a.part[(b * a.rows + j) * a.pieces + lane] : Piece{0.0, -__builtin_inff(), INT32_MAX};
    m = p.top;
    s = p.sum;
    arg = p.arg;
    for (int d = 32; d > 0; d >>= 1) {
        const float m2 = __shfl_xor(m, d);
        const int arg2 = __shfl_xor(arg, d);
        larger(m, arg, m2, arg2);
    }
    if (c != 0.0) s *= exp2_64((p.top - double(finite_ref(m))) * c);
    for (int d = 32; d > 0; d >>= 1) s += __shfl_xor(s, d);
}

// Whether a row has a probability to draw from.
__device__ __forceinline__ bool good_sum(double s) { return s > 0.0 && s < __builtin_inf(); }

struct DecideShared {
    float m[2 * MAXL + 1];
    double s[2 * MAXL + 1];
    int arg[MAXL + 1];
    int count, bad;
};

// Which drafts are accepted, by the whole block. (Ends with a barrier.)
template <bool PB, bool QB>
__device__ __forceinline__ Decision decide(const DArgs &a, int64_t b, DecideShared &sh)
{
    const int t = threadIdx.x, lane = t & 63, w = t >> 6;
    bool bad = false;
    const int n = seq_len(a, b, bad);
    const double c = seq_scale(a, b, bad);
    for (int j = w; j < a.rows; j += DT / 64) {
        const bool target = j <= a.L;
        const int i = target ? j : j - a.L - 1;
        if (target ? i > n : (i >= n || c == 0.0)) continue;
        float m;
        double s;
        int arg;
        row_stats(a, b, j, c, m, s, arg);
        if (lane == 0) {
            sh.m[j] = m;
            sh.s[j] = s;
            if (target) sh.arg[i] = arg;
        }
    }
    __syncthreads();
    if (w == 0) {
        bool ok = false;
        if (lane < n) {
            const int x = a.tokens[b * a.L + lane];
            if (x < 0 || x >= a.N) {
                bad = true;
            } else if (c == 0.0) {
                ok = x == sh.arg[lane] && sh.s[lane] == 0.0;
            } else {
                const Rows<PB, QB> rows(a, b, lane);
                const double p = exp2_64((word_at<PB>(rows.p, x) - double(finite_ref(sh.m[lane]))) * c) / sh.s[lane];
                double q = 1.0;
                if (a.Q) {
                    const int j = a.L + 1 + lane;
                    q = exp2_64((word_at<QB>(rows.q, x) - double(finite_ref(sh.m[j]))) * c) / sh.s[j];
                }
                ok = double(a.u[b * a.L + lane]) * q < p;
            }
        }
        const uint64_t no = ~__ballot(ok);
        const uint64_t any = __ballot(bad);
        if (lane == 0) {
            const int first = no ? __builtin_ctzll(no) : 64;
            sh.count = first < n ? first : n;
            sh.bad = any != 0;
        }
    }
    __syncthreads();
    Decision d;
    d.count = sh.count;
    d.mp = sh.m[d.count];
    d.sp = sh.s[d.count];
    d.arg = sh.arg[d.count];
    d.mq = 0.0f;
    d.sq = 1.0;
    d.token = d.count < n ? a.tokens[b * a.L + d.count] : -1;
    d.bits = sh.bad ? BSQ_DEVERR_BAD_SET : 0;
    d.pad = 0;
    if (c == 0.0) {
        d.kind = d.sp == 0.0 && d.arg != INT32_MAX ? DRAW_LARGEST : DRAW_NONE;
    } else if (!good_sum(d.sp)) {
        d.kind = DRAW_NONE;
    } else if (d.count == n) {
        d.kind = DRAW_TARGET;
    } else if (!a.Q) {
        d.kind = DRAW_OTHERS;
    } else {
        const int j = a.L + 1 + d.count;
        d.mq = sh.m[j];
        d.sq = sh.s[j];
        d.kind = good_sum(d.sq) ? DRAW_REST : DRAW_TARGET;
        if (d.kind == DRAW_TARGET) d.bits |= BSQ_DEVERR_NONFINITE;
    }
    if (d.kind == DRAW_NONE) d.bits |= BSQ_DEVERR_NONFINITE;
    return d;
}

// The weight of word i in the draw.
struct Weight {
    double c, mp, mq, ip, iq;
    int kind;
    int64_t token;
    __device__ __forceinline__ Weight(const Decision &d, double scale)
        : c(scale), mp(d.mp), mq(d.mq), ip(1.0 / d.sp), iq(1.0 / d.sq), kind(d.kind), token(d.token)
    {
    }
    __device__ __forceinline__ double operator()(float zp, float zq, int64_t i) const
    {
        const double p = exp2_64((zp - mp) * c);
        if (kind == DRAW_TARGET) return p;
        if (kind == DRAW_OTHERS) return i == token ? 0.0 : p;
        const double q = exp2_64((zq - mq) * c);
        const double d = p * ip - q * iq;
        return d > 0.0 ? d : 0.0;
    }
};

__device__ __forceinline__ double block_sum64(double v, double *s)
{
    const int t = threadIdx.x, lane = t & 63;
    for (int d = 32; d > 0; d >>= 1) v += __shfl_xor(v, d);
    if (lane == 0) s[t >> 6] = v;
    __syncthreads();
    v = 0.0;
    for (int w = 0; w < DT / 64; ++w) v += s[w];
    __syncthreads();
    return v;
}

// Decisions, and the weight of every piece of the row that the next token is drawn from.
template <bool PB, bool QB>
__global__ __launch_bounds__(DT) void draft_rest_kernel(const DArgs a)
{
    __shared__ DecideShared sh;
    __shared__ double s_sum[DT / 64];
    const int t = threadIdx.x;
    const int64_t items = a.B * a.pieces;
    for (int64_t item = blockIdx.x; item < items; item += gridDim.x) {
        const int64_t b = item / a.pieces, piece = item - b * a.pieces;
        const Decision d = decide<PB, QB>(a, b, sh);
        if (piece == 0 && t == 0) {
            a.dec[b] = d;
            if (d.bits && a.err) atomicOr(a.err, d.bits);
        }
        if (d.kind != DRAW_LARGEST && d.kind != DRAW_NONE) {
            bool bad = false;
            const Weight weight(d, seq_scale(a, b, bad));
            const int64_t n0 = piece * a.len, n1 = n0 + a.len < a.N ? n0 + a.len : a.N;
            const bool again = d.kind == DRAW_REST || (d.kind == DRAW_OTHERS && d.token >= n0 && d.token < n1);
            double s = 0.0;
            if (again) {
                const Rows<PB, QB> rows(a, b, d.count);
                const bool rest = d.kind == DRAW_REST;
                for (int64_t base = n0 + 8 * t; base < n1; base += 2 * VSTEP) {
                    Words8<PB> p[2];
                    Words8<QB> q[2];
#pragma unroll
                    for (int k = 0; k < 2; ++k) {
                        const int64_t at = base + k * VSTEP < n1 ? base + k * VSTEP : n1;
                        p[k].load(rows.p, at, n1);
                        if (rest) q[k].load(rows.q, at, n1);
                    }
#pragma unroll
                    for (int k = 0; k < 2; ++k)
#pragma unroll
                        for (int e = 0; e < 8; ++e) s += weight(p[k][e], rest ? q[k][e] : 0.0f, base + k * VSTEP + e);
                }
                s = block_sum64(s, s_sum);
            } else {
                const Piece p = a.part[(b * a.rows + d.count) * a.pieces + piece];
                s = p.sum * exp2_64((p.top - double(d.mp)) * weight.c);
            }
            if (t == 0) a.rest[item] = s;
        }
        __syncthreads();
    }
}

// Inclusive sums over a wave.
__device__ __forceinline__ double wave_scan(double v)
{
    const int lane = threadIdx.x & 63;
    for (int d = 1; d < 64; d <<= 1) {
        const double o = __shfl_up(v, d);
        if (lane >= d) v += o;
    }
    return v;
}

// The draw and the outputs: a block a sequence.
template <bool PB, bool QB>
__global__ __launch_bounds__(DT) void draft_draw_kernel(const DArgs a)
{
    __shared__ double s_sum[DT / 64], s_target, s_before;
    __shared__ int s_piece, s_kind, s_first;
    __shared__ unsigned s_last;
    const int t = threadIdx.x, lane = t & 63, w = t >> 6;
    const int64_t b = blockIdx.x;
    Decision d = a.dec[b];
    bool bad = false;
    const double c = seq_scale(a, b, bad);
    if (w == 0) {
        // the piece where the cumulative sum passes r times the whole
        double v = lane < a.pieces && d.kind <= DRAW_OTHERS ? a.rest[b * a.pieces + lane] : 0.0;
        double incl = wave_scan(v), all = __shfl(incl, 63);
        int kind = d.kind;
        if ((kind == DRAW_REST || kind == DRAW_OTHERS) && !good_sum(all)) {
            // nothing is left beside what was refused (p and q differ by roundings alone)
            kind = DRAW_TARGET;
            v = 0.0;
            if (lane < a.pieces) {
                const Piece p = a.part[(b * a.rows + d.count) * a.pieces + lane];
                v = p.sum * exp2_64((p.top - double(d.mp)) * c);
            }
            incl = wave_scan(v);
            all = __shfl(incl, 63);
        }
        const double r = a.r[b], target = r * all;
        const uint64_t past = __ballot(incl > target), some = __ballot(v > 0.0);
        const uint64_t in = past & some;
        const int piece = in ? __builtin_ctzll(in) : (some ? 63 - __builtin_clzll(some) : 0);
        const double before = __shfl(incl - v, piece);
        if (lane == 0) {
            s_piece = piece;
            s_kind = kind;
            s_target = target;
            s_before = before;
            s_last = 0u;
        }
    }
    __syncthreads();
    d.kind = s_kind;
    int next = -1;
    if (d.kind == DRAW_LARGEST) {
        next = d.arg;
    } else if (d.kind != DRAW_NONE) {
        const Weight weight(d, c);
        const Rows<PB, QB> rows(a, b, d.count);
        const bool rest = d.kind == DRAW_REST;
        const int64_t n0 = int64_t(s_piece) * a.len, n1 = n0 + a.len < a.N ? n0 + a.len : a.N;
        double before = s_before;
        const double target = s_target;
        // runs of eight words a thread, in order
        for (int64_t base = n0; base < n1 && next < 0; base += VSTEP) {
            const int64_t at = base + 8 * t < n1 ? base + 8 * t : n1;
            Words8<PB> p;
            Words8<QB> q;
            p.load(rows.p, at, n1);
            if (rest) q.load(rows.q, at, n1);
            double v[8], own = 0.0;
            int last = -1;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                v[e] = weight(p[e], rest ? q[e] : 0.0f, at + e);
                own += v[e];
                if (v[e] > 0.0) last = e;
            }
            const double scan = wave_scan(own);
            if (lane == 63) s_sum[w] = scan;
            if (t == 0) s_first = DT;
            __syncthreads();
            double at0 = before, whole = before;
            for (int k = 0; k < DT / 64; ++k) {
                if (k < w) at0 += s_sum[k];
                whole += s_sum[k];
            }
            if (last >= 0) {
                atomicMax(&s_last, unsigned(at + last));
                if (at0 + scan > target) atomicMin(&s_first, t);
            }
            __syncthreads();
            const int first = s_first;
            if (first < DT) {
                if (t == first) {
                    double sum = at0 + (scan - own);
                    int pick = -1;
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        sum += v[e];
                        if (pick < 0 && sum > target && v[e] > 0.0) pick = e;
                    }
                    s_last = unsigned(at + (pick < 0 ? last : pick));
                }
                __syncthreads();
                next = int(s_last);
            }
            before = whole;
            __syncthreads();
        }
        // (roundings: the piece's words add up to less than its sum by the first pass)
        if (next < 0) next = int(s_last);
    }
    for (int i = t; i <= a.L; i += DT)
        a.out[b * (a.L + 1) + i] = i < d.count ? a.tokens[b * a.L + i] : (i == d.count ? next : -1);
    if (t == 0) a.count[b] = d.count;
}

// ---------------------------------------------------------------------------
// Host side.
// ---------------------------------------------------------------------------
struct DLayout {
    int rows, pieces;
    int64_t len;
    size_t part, rest, dec, total;
};

DLayout draft_layout(int64_t B, int64_t L, int64_t N, bool draft)
{
    DLayout l{};
    l.rows = int(L + 1 + (draft ? L : 0));
    // pieces of whole steps of a block, at most one a lane
    const int64_t steps = (N + VSTEP - 1) / VSTEP;
    const int64_t most = NV;  // steps that a thread reads together
    int64_t per = std::max<int64_t>((steps + MAX_PIECES - 1) / MAX_PIECES, most);
    l.len = per * VSTEP;
    l.pieces = int((N + l.len - 1) / l.len);
    size_t at = 0;
    auto take = [&](size_t bytes) {
        const size_t p = at;
        at += align256(bytes);
        return p;
    };
    l.part = take(size_t(B) * l.rows * l.pieces * sizeof(Piece));
    l.rest = take(size_t(B) * l.pieces * sizeof(double));
    l.dec = take(size_t(B) * sizeof(Decision));
    l.total = at;
    return l;
}

template <bool PB, bool QB>
hipError_t launch_draft(const DArgs &a, hipStream_t st)
{
    const int64_t most = int64_t(1) << 20;  // blocks of a launch; they walk the rest
    hipLaunchKernelGGL((draft_rows_kernel<PB, QB>), dim3(unsigned(std::min(most, a.B * a.rows * a.pieces))), dim3(DT), 0, st, a);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((draft_rest_kernel<PB, QB>), dim3(unsigned(std::min(most, a.B * a.pieces))), dim3(DT), 0, st, a);
    if ((e = hipGetLastError()) != hipSuccess) return e;
    hipLaunchKernelGGL((draft_draw_kernel<PB, QB>), dim3(unsigned(a.B)), dim3(DT), 0, st, a);
    return hipGetLastError();
}

}  // namespace

size_t draft_ws_bytes(int64_t B, int64_t L, int64_t N, bool draft) { return draft_layout(B, L, N, draft).total; }

hipError_t launch_draft_verify(const DraftCall &c, hipStream_t st)
{
    const DLayout l = draft_layout(c.B, c.L, c.N, c.Q != nullptr);
    char *ws = static_cast<char *>(c.ws);
    DArgs a{};
    a.P = c.P;
    a.Q = c.Q;
    a.B = c.B;
    a.N = c.N;
    a.pseq = c.pseq;
    a.prow = c.prow;
    a.qseq = c.qseq;
    a.qrow = c.qrow;
    a.L = int(c.L);
    a.rows = l.rows;
    a.pieces = l.pieces;
    a.len = l.len;
    a.tokens = c.tokens;
    a.lens = c.lens;
    a.u = c.u;
    a.r = c.r;
    a.temp = c.temp;
    a.count = c.count;
    a.out = c.out;
    a.err = c.err;
    a.part = reinterpret_cast<Piece *>(ws + l.part);
    a.rest = reinterpret_cast<double *>(ws + l.rest);
    a.dec = reinterpret_cast<Decision *>(ws + l.dec);
    const bool pb = c.p_dtype == BSQ_BF16, qb = c.Q ? c.q_dtype == BSQ_BF16 : pb;
    if (pb) return qb ? launch_draft<true, true>(a, st) : launch_draft<true, false>(a, st);
    return qb ? launch_draft<false, true>(a, st) : launch_draft<false, false>(a, st);
}

}  // namespace bsq
