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
// Three launches: the largest logit and the sum of exponentials of every row that is
// needed; the weights of the one row that the next token is drawn from, summed over runs of
// 512 words (every block first decides its sequence from the first launch's results); the
// draw, a wave a sequence. No atomics but an OR of error bits: a result depends on the
// inputs alone.
//
// Results are those of 64-bit sums. A cumulative sum over 151936 words passes a given
// random number at the same word as the definition's only if it is off by much less than
// one word's share; with exponentials of 32 bits (some 3e-8 of the sum off) one draw in
// some 200 would be another word. Exponentials of 64 bits bound the reading (all rows of 64
// sequences 78 us, in 32 bits 39), so the rows that only decide are summed in 32 (3e-5 of a
// ratio covers every rounding), and where u q lies so near to p that this does not settle
// it the block sums the two rows again in 64. max(p - q, 0) of the drawn row needs both
// rows' sums before it can be formed: the second launch instead splits p and q into the
// words where p is larger, by the first launch's sums, and their rests, and marks the runs
// that hold a word where p / q lies within 2^-20 of 1. The draw puts them together with the
// exact sums, which are by now known to say how far off the first ones were (up to 5e-7 in
// 2600 rows of many shapes): where that is less than 2^-20 only the marked runs can hold a word on
// the wrong side, and their weights are formed anew, word by word; else those of all.
//
// 64 sequences of four drafts, 151936 words in bf16: rows 39 us (175 MB, 4.5 TB/s), the
// drawn rows 35 to 36 (64-bit exponentials: two a word), draws 7 to 8. One sequence: 6, 9 and 6, each
// a chain of a few dependent loads. Where all runs are weighed anew (drafts in bf16 that
// are the target's but for some words) the draws take some 350 more: a wave reads both
// rows.
#include <algorithm>

#include "vocab_rows.h"

namespace bsq {
namespace {

constexpr int DT = 256;                // threads of a block
constexpr int64_t VSTEP = 8 * DT;      // words of a vector a thread
constexpr int64_t MOST_TURNS = 2048;   // blocks of the first launch: those that run together
constexpr int64_t MAX_RUNS = 4096;     // of a row: 64 a lane
constexpr int64_t RUN = 512;           // words of a vector a lane
constexpr int MAXL = BSQ_MAX_DRAFTS;
constexpr double LOG2E_64 = 1.4426950408889634074;
constexpr float MAX_TEMPERATURE = 0x1p64f, MIN_TEMPERATURE = 0x1p-64f;
// Of p, what the first launch's sums leave open. A term's exponent is rounded three times
// (2^-24 of it each; its mean under the softmax is at most log2 N < 31), the exponential by
// 2^-22, a thread's 32 terms by 2^-19: 8e-6 of a sum, 1.6e-5 of the ratio of two. And in every
// turn that a block has of a row a larger logit may rescale what came before, by an exponential
// that is 2^-22 off.
constexpr double UNSURE = 0x1p-15, UNSURE_TURN = 0x1p-21;
// Of p, how near q has to be for the first launch's sums to leave open which is larger: 2^-20.
// (Few words are: of drafts with noise of 0.6 in their logits one in 10^6.)
constexpr int CLOSE_BITS = 20;
constexpr double CLOSE = 0x1p-20;
static_assert(MAXL <= 64, "a lane for every drafted token");
static_assert(2 * MAXL + 1 <= DT, "a thread for every row");

enum { DRAW_TARGET, DRAW_REST, DRAW_OTHERS, DRAW_LARGEST, DRAW_NONE };

struct Piece {
    double sum;   // of 32-bit exponentials against `top` (greedy rows: 0, or NaN where a logit is)
    float top;
    int32_t arg;  // greedy rows: lowest index of the largest
};

// Of a run of the row that is drawn from: its words' exponentials (without the refused token
// of a certain draft) and the draft row's, and of both those of the words where p > q by the
// first launch's sums; close: whether it has words where those leave this open.
struct Run {
    double p, q, above_p, above_q;
    int32_t close, pad;
};

// What a sequence's drafts came to: `kind` of draw, the rows' largest logits and sums (those
// of the first launch).
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
    int L, rows;          // rows: of a sequence, L + 1 (+ L with draft logits)
    int64_t turn, turns;  // words of a block's turn; turns of a row
    int64_t per;          // turns of a block: those of all rows one after another
    int64_t pieces;       // parts of a row that blocks have, at most
    double unsure;        // of p: what their sums leave open
    int64_t run;          // words of a run
    int runs, parts;      // of a row; blocks that share a row's runs
    const int32_t *tokens, *lens;
    const float *u, *r, *temp;
    int32_t *count, *out, *err;
    Piece *part;          // [B][rows][pieces]
    Run *rest;            // [B][runs]
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

// log2(e) over the temperature; 0 for a greedy sequence, one below 2^-64 among them. (A
// temperature that is negative, NaN or above 2^64 is reported and counts as 0.)
__device__ __forceinline__ double seq_scale(const DArgs &a, int64_t b, bool &bad)
{
    if (!a.temp) return LOG2E_64;
    const float t = a.temp[b];
    if (!(t >= 0.0f && t <= MAX_TEMPERATURE)) {
        bad = true;
        return 0.0;
    }
    return t < MIN_TEMPERATURE ? 0.0 : LOG2E_64 / double(t);
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

// The larger of two, of equal ones the lower index.
__device__ __forceinline__ void larger(float &m, int &arg, float m2, int arg2)
{
    if (m2 > m || (m2 == m && arg2 < arg)) {
        m = m2;
        arg = arg2;
    }
}

// A thread's largest logit (greedy: and its lowest index) and sum over words [n0, n1) of
// a row, NV vectors at a time, the next ones in flight.
template <bool BF16, int NV>
__device__ __forceinline__ void piece_stats(const void *row, int64_t n0, int64_t n1, float c, float &m, double &s, int &arg)
{
    m = -__builtin_inff();
    s = 0.0;
    arg = INT32_MAX;
    Words8<BF16> next[NV];
    auto load = [&](int64_t base) {
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const int64_t at = base + k * VSTEP;
            next[k].load(row, at < n1 ? at : n1, n1);
        }
    };
    load(n0 + 8 * threadIdx.x);
    // Every thread has the same turns: one whose words of the last lie past n1 has -inf there.
    for (int64_t turn = n0; turn < n1; turn += NV * VSTEP) {
        const int64_t base = turn + 8 * threadIdx.x;
        Words8<BF16> w[NV];
#pragma unroll
        for (int k = 0; k < NV; ++k) w[k] = next[k];
        if (turn + NV * VSTEP < n1) load(base + NV * VSTEP);
        if (c == 0.0f) {
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
        // (taken apart again for the sum: kept, the words would take twice the registers)
#pragma unroll
        for (int k = 0; k < NV; ++k)
#pragma unroll
            for (int h = 0; h < int(sizeof(w[0].raw) / 16); ++h) asm volatile("" : "+v"(w[k].raw[h]));
        const float ref = mx == -__builtin_inff() ? 0.0f : mx;
        if (mx > m) {
            s *= double(__builtin_amdgcn_exp2f((m - ref) * c));
            m = mx;
        }
        float sum = 0.0f;
#pragma unroll
        for (int k = 0; k < NV; ++k)
#pragma unroll
            for (int e = 0; e < 8; ++e) sum += __builtin_amdgcn_exp2f((w[k][e] - ref) * c);
        s += double(sum);
    }
}

// Largest logit and sum of every row that the sequences need: the turns of all rows, in
// equal shares; a block leaves one piece of every row that it has turns of.
template <bool PB, bool QB, int NV>
__global__ __launch_bounds__(DT) void draft_rows_kernel(const DArgs a)
{
    __shared__ float s_m[DT / 64];
    __shared__ double s_s[DT / 64];
    __shared__ int s_arg[DT / 64];
    const int t = threadIdx.x, lane = t & 63, w = t >> 6;
    const int64_t all = a.B * a.rows * a.turns;
    const int64_t x0 = blockIdx.x * a.per, x1 = x0 + a.per < all ? x0 + a.per : all;
    for (int64_t x = x0; x < x1;) {
        const int64_t rr = x / a.turns, b = rr / a.rows;
        const int j = int(rr - b * a.rows);
        const int64_t first = x - rr * a.turns, end = x1 < (rr + 1) * a.turns ? x1 : (rr + 1) * a.turns;
        const int64_t count = end - x;
        x = end;
        bool bad = false;
        const int n = seq_len(a, b, bad);
        const double c = seq_scale(a, b, bad);
        const bool target = j <= a.L;
        const int i = target ? j : j - a.L - 1;
        if (target ? i > n : (i >= n || c == 0.0)) continue;
        const Rows<PB, QB> rows(a, b, i);
        const int64_t n0 = first * a.turn, n1 = n0 + count * a.turn < a.N ? n0 + count * a.turn : a.N;
        const double reach = 1000.0 / c;
        float m;
        double s;
        int arg;
        if (target) piece_stats<PB, NV>(rows.p, n0, n1, float(c), m, s, arg);
        else piece_stats<QB, NV>(rows.q, n0, n1, float(c), m, s, arg);
        float wm = wave_max(m);
        // (the lowest index among the lanes that hold the largest)
        if (c == 0.0) arg = lane_value(wave_scan(m == wm ? arg : INT32_MAX, INT32_MAX, [](int x, int y) { return x < y ? x : y; }), 63);
        if (c != 0.0) s *= Exp2Below(wm, c, reach)(m);
        s = wave_sum(s);
        if (lane == 0) {
            s_m[w] = wm;
            s_s[w] = s;
            s_arg[w] = arg;
        }
        __syncthreads();
        if (t == 0) {
            float m0 = wm;
            for (int k = 1; k < DT / 64; ++k) larger(wm, arg, s_m[k], s_arg[k]);
            if (c != 0.0) {
                const Exp2Below e2(wm, c, reach);
                s *= e2(m0);
                for (int k = 1; k < DT / 64; ++k) s += s_s[k] * e2(s_m[k]);
            } else {
                for (int k = 1; k < DT / 64; ++k) s += s_s[k];
            }
            a.part[rr * a.pieces + (blockIdx.x - rr * a.turns / a.per)] = Piece{s, wm, arg};
        }
        __syncthreads();
    }
}

// Whether a row has a probability to draw from.
__device__ __forceinline__ bool good_sum(double s) { return s > 0.0 && s < __builtin_inf(); }

struct DecideShared {
    float m[2 * MAXL + 1];
    double s[2 * MAXL + 1];
    int arg[MAXL + 1];
    double sum[DT / 64];
    int count, bad, ask;
};

// Sum of exponentials of a whole row in 64 bits, by the block. (Two barriers.)
template <bool BF16>
__device__ __forceinline__ double row_sum(const void *row, int64_t N, float m, double c, double reach, double *s_sum)
{
    const int t = threadIdx.x;
    const Exp2Below e2(m, c, reach);
    double s = 0.0;
    for (int64_t at = 8 * t; at < N; at += VSTEP) {
        Words8<BF16> w;
        w.load(row, at, N);
#pragma unroll
        for (int e = 0; e < 8; ++e) s += e2(w[e]);
    }
    s = wave_sum(s);
    if ((t & 63) == 0) s_sum[t >> 6] = s;
    __syncthreads();
    s = 0.0;
    for (int w = 0; w < DT / 64; ++w) s += s_sum[w];
    __syncthreads();
    return s;
}

// Which drafts are accepted, by the whole block: some lanes join the pieces of a row, a lane
// of the first wave decides a token. (Ends with a barrier.)
template <bool PB, bool QB>
__device__ __forceinline__ Decision decide(const DArgs &a, int64_t b, int n, double c, double reach, bool bad,
                                           DecideShared &sh)
{
    const int t = threadIdx.x;
    // what the decisions need of the tokens, read ahead of the join
    int x = -1;
    float u = 0.0f, zp = 0.0f, zq = 0.0f;
    if (t < n) {
        x = a.tokens[b * a.L + t];
        u = a.u[b * a.L + t];
        if (x < 0 || x >= a.N) {
            bad = true;
            x = -1;
        } else if (c != 0.0) {
            const Rows<PB, QB> rows(a, b, t);
            zp = word_at<PB>(rows.p, x);
            if (a.Q) zq = word_at<QB>(rows.q, x);
        }
    }
    // up to 16 lanes a row
    int log = 0;
    while (log < 4 && (a.rows << (log + 1)) <= DT) ++log;
    const int j = t >> log, lanes = 1 << log, g = t & (lanes - 1);
    const bool target = j <= a.L;
    const int i = target ? j : j - a.L - 1;
    const bool need = j < a.rows && (target ? i <= n : (i < n && c != 0.0));
    {
        const int64_t rr = b * a.rows + j;
        const Piece *p = a.part + rr * a.pieces;
        const int end = need ? int(((rr + 1) * a.turns - 1) / a.per - rr * a.turns / a.per + 1) : 0;
        float m = -__builtin_inff();
        double s = 0.0;
        int arg = INT32_MAX;
#pragma unroll 4
        for (int k = g; k < end; k += lanes) larger(m, arg, p[k].top, p[k].arg);
        for (int d = lanes >> 1; d > 0; d >>= 1) {
            const float m2 = __shfl_xor(m, d);
            const int arg2 = __shfl_xor(arg, d);
            larger(m, arg, m2, arg2);
        }
        const Exp2Below e2(m, c, reach);
#pragma unroll 4
        for (int k = g; k < end; k += lanes) s += c != 0.0 ? p[k].sum * e2(p[k].top) : p[k].sum;
        for (int d = lanes >> 1; d > 0; d >>= 1) s += __shfl_xor(s, d);
        if (need && g == 0) {
            sh.m[j] = m;
            sh.s[j] = s;
            if (target) sh.arg[i] = arg;
        }
    }
    __syncthreads();
    bool ok = false, unsure = false;
    const int jq = a.L + 1 + t;
    if (x >= 0) {
        if (c == 0.0) {
            ok = x == sh.arg[t] && sh.s[t] == 0.0;
        } else {
            const double p = Exp2Below(sh.m[t], c, reach)(zp) / sh.s[t];
            const double q = a.Q ? Exp2Below(sh.m[jq], c, reach)(zq) / sh.s[jq] : 1.0;
            ok = double(u) * q < p;
            unsure = p > 0.0 && __builtin_fabs(double(u) * q - p) <= a.unsure * p;
        }
    }
    for (;;) {
        if (t < 64) {
            const uint64_t stop = ~__ballot(ok && !unsure), any = __ballot(bad), open = __ballot(unsure);
            if (t == 0) {
                const int first = stop ? __builtin_ctzll(stop) : 64;
                sh.count = first < n ? first : n;
                sh.ask = first < n && ((open >> first) & 1);
                sh.bad = any != 0;
            }
        }
        __syncthreads();
        if (!sh.ask) break;
        // by the rows' sums in 64 bits
        const int k = sh.count;
        const Rows<PB, QB> rows(a, b, k);
        const double sp = row_sum<PB>(rows.p, a.N, sh.m[k], c, reach, sh.sum);
        const double sq = a.Q ? row_sum<QB>(rows.q, a.N, sh.m[a.L + 1 + k], c, reach, sh.sum) : 1.0;
        if (t == k) {
            const double p = Exp2Below(sh.m[t], c, reach)(zp) / sp;
            const double q = a.Q ? Exp2Below(sh.m[jq], c, reach)(zq) / sq : 1.0;
            ok = double(u) * q < p;
            unsure = false;
        }
    }
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
        d.mq = sh.m[a.L + 1 + d.count];
        d.sq = sh.s[a.L + 1 + d.count];
        d.kind = good_sum(d.sq) ? DRAW_REST : DRAW_TARGET;
        if (d.kind == DRAW_TARGET) d.bits |= BSQ_DEVERR_NONFINITE;
    }
    if (d.kind == DRAW_NONE) d.bits |= BSQ_DEVERR_NONFINITE;
    return d;
}

// Exponentials of the row that is drawn from, and of the draft's where `rest` is asked for.
template <bool PB, bool QB>
struct Drawn {
    Rows<PB, QB> rows;
    Exp2Below p, q;
    int64_t out;  // the word that is left out, or -1
    __device__ __forceinline__ Drawn(const DArgs &a, int64_t b, const Decision &d, double c, double reach)
        : rows(a, b, d.count), p(d.mp, c, reach), q(d.mq, c, reach), out(d.kind == DRAW_OTHERS ? d.token : -1)
    {
    }
    // eight words from `at` on (-inf past `end`)
    __device__ __forceinline__ void read(int64_t at, int64_t end, bool rest, Words8<PB> &zp, Words8<QB> &zq) const
    {
        zp.load(rows.p, at < end ? at : end, end);
        if (rest) zq.load(rows.q, at < end ? at : end, end);
    }
    __device__ __forceinline__ void eight(int64_t at, int64_t end, bool rest, double (&ep)[8], double (&eq)[8]) const
    {
        Words8<PB> zp;
        Words8<QB> zq;
        read(at, end, rest, zp, zq);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            ep[e] = p(zp[e]);
            if (at + e == out) ep[e] = 0.0;
            eq[e] = rest ? q(zq[e]) : 0.0;
        }
    }
};

__device__ __forceinline__ int32_t high_word(double v) { return int32_t(__builtin_bit_cast(uint64_t, v) >> 32); }

// Decisions, and the weight of every run of the row that the next token is drawn from.
template <bool PB, bool QB>
__global__ __launch_bounds__(DT) void draft_rest_kernel(const DArgs a)
{
    __shared__ DecideShared sh;
    const int t = threadIdx.x, lane = t & 63, w = t >> 6;
    const uint32_t b = blockIdx.x / uint32_t(a.parts), part = blockIdx.x - b * a.parts;
    bool bad = false;
    const int n = seq_len(a, b, bad);
    const double c = seq_scale(a, b, bad);
    const double reach = 1000.0 / c;
    const Decision d = decide<PB, QB>(a, b, n, c, reach, bad, sh);
    if (part == 0 && t == 0) {
        a.dec[b] = d;
        if (d.bits && a.err) atomicOr(a.err, d.bits);
    }
    if (d.kind <= DRAW_OTHERS) {
        const Drawn<PB, QB> drawn(a, b, d, c, reach);
        const bool rest = d.kind == DRAW_REST;
        const double ratio = d.sp / d.sq;  // p > q where ep > eq ratio
        // (vectors of a wave: the next one is in flight)
        Words8<PB> zp;
        Words8<QB> zq;
        const int step = a.parts * (DT / 64);
        int r = part * (DT / 64) + w;
        auto read = [&](int run, int64_t at) {
            const int64_t n0 = run * a.run, n1 = n0 + a.run < a.N ? n0 + a.run : a.N;
            drawn.read(n0 + at + 8 * lane, n1, rest, zp, zq);
        };
        if (r < a.runs) read(r, 0);
        for (; r < a.runs; r += step) {
            const int64_t n0 = r * a.run;
            Run s{0.0, 0.0, 0.0, 0.0, 0, 0};
            int32_t closest = 0;  // how far the high word of ep - eq ratio is below that of ep
            for (int64_t at = 0; at < a.run; at += RUN) {
                const Words8<PB> wp = zp;
                const Words8<QB> wq = zq;
                if (at + RUN < a.run) read(r, at + RUN);
                else if (r + step < a.runs) read(r + step, 0);
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const double ep = n0 + at + 8 * lane + e == drawn.out ? 0.0 : drawn.p(wp[e]);
                    s.p += ep;
                    if (!rest) continue;
                    const double eq = drawn.q(wq[e]);
                    // (by the high words: exponent and 20 bits. Equal ones count as above and are
                    // close, those of 0 add nothing and are not)
                    const int32_t more = high_word(__builtin_fma(-eq, ratio, ep)), below = high_word(ep) - (more & 0x7fffffff);
                    const bool above = more >= 0;
                    closest = below > closest ? below : closest;
                    s.q += eq;
                    s.above_p += above ? ep : 0.0;
                    s.above_q += above ? eq : 0.0;
                }
            }
            s.p = wave_sum(s.p);
            if (rest) {
                s.q = wave_sum(s.q);
                s.above_p = wave_sum(s.above_p);
                s.above_q = wave_sum(s.above_q);
                s.close = __ballot(closest > (CLOSE_BITS << 20)) != 0;
            }
            if (lane == 0) a.rest[int64_t(b) * a.runs + r] = s;
        }
    }
}

__device__ __forceinline__ double sum_scan(double v)
{
    return wave_scan(v, 0.0, [](double x, double y) { return x + y; });
}

// The first lane whose cumulative sum `incl` exceeds `target` and that holds some of it;
// the last one that holds some where roundings leave none; -1 where no lane holds any.
__device__ __forceinline__ int crossing(double incl, double own, double target)
{
    const uint64_t some = __ballot(own > 0.0), past = __ballot(incl > target) & some;
    return past ? __builtin_ctzll(past) : (some ? 63 - __builtin_clzll(some) : -1);
}

// The draw and the outputs: a wave a sequence.
template <bool PB, bool QB>
__global__ __launch_bounds__(64) void draft_draw_kernel(const DArgs a)
{
    const int lane = threadIdx.x;
    const int64_t b = blockIdx.x;
    Decision d = a.dec[b];
    bool bad = false;
    const double c = seq_scale(a, b, bad), r = a.r[b];
    int next = -1;
    if (d.kind == DRAW_LARGEST) {
        next = d.arg;
    } else if (d.kind != DRAW_NONE) {
        // every lane `per` runs in order
        const int per = (a.runs + 63) / 64, r0 = lane * per, r1 = r0 + per < a.runs ? r0 + per : a.runs;
        Run *runs = a.rest + b * a.runs;
        double ip = 1.0, iq = 0.0;  // a word's weight: ep ip - eq iq, where that is more than 0
        bool rest = d.kind == DRAW_REST;
        const Drawn<PB, QB> drawn(a, b, d, c, 1000.0 / c);
        uint64_t open = 0;  // the lane's runs that may hold a word on the wrong side
        if (rest) {
            double sp = 0.0, sq = 0.0;
#pragma unroll 4
            for (int k = r0; k < r1; ++k) {
                sp += runs[k].p;
                sq += runs[k].q;
                open |= uint64_t(runs[k].close) << (k - r0);
            }
            ip = 1.0 / wave_sum(sp);
            iq = 1.0 / wave_sum(sq);
            // (2^-10 of it for the roundings of this comparison and of the marks)
            if (!(__builtin_fabs(d.sp / d.sq * ip / iq - 1.0) < CLOSE * (1.0 - 0x1p-10)))
                open = r0 < r1 ? ~uint64_t(0) >> (64 - (r1 - r0)) : 0;
        }
        auto weight = [&](double ep, double eq) {
            const double v = ep * ip - eq * iq;
            return v > 0.0 ? v : 0.0;
        };
        auto run_weight = [&](int k) { return rest ? weight(runs[k].above_p, runs[k].above_q) : runs[k].p; };
        auto lane_weight = [&]() {
            double v = 0.0;
#pragma unroll 4
            for (int k = r0; k < r1; ++k) v += run_weight(k);
            return v;
        };
        // their weights word by word; the lane that has the run keeps it
        for (uint64_t some; (some = __ballot(open != 0)) != 0;) {
            const int who = __builtin_ctzll(some), run = lane_value(r0 + (open ? __builtin_ctzll(open) : 0), who);
            const int64_t n0 = run * a.run, n1 = n0 + a.run < a.N ? n0 + a.run : a.N;
            double s = 0.0;
            for (int64_t at = n0; at < n1; at += RUN) {
                double ep[8], eq[8];
                drawn.eight(at + 8 * lane, n1, true, ep, eq);
#pragma unroll
                for (int e = 0; e < 8; ++e) s += weight(ep[e], eq[e]);
            }
            s = wave_sum(s);
            if (lane == who) {
                runs[run].above_p = s / ip;
                runs[run].above_q = 0.0;
                open &= open - 1;
            }
        }
        double own = lane_weight(), incl = sum_scan(own), all = lane_value(incl, 63);
        if (rest && !good_sum(all)) {
            // nothing is left beside what was refused: p itself
            rest = false;
            ip = 1.0;
            iq = 0.0;
            own = lane_weight();
            incl = sum_scan(own);
            all = lane_value(incl, 63);
        }
        if (!good_sum(all)) {
            next = d.token;  // (the refused token is all that p holds)
        } else {
            const double target = r * all;
            const int who = crossing(incl, own, target);
            // that lane's first run past it (roundings: its last run with a weight)
            double sum = incl - own, at_run = sum, at_last = sum;
            int run = -1, some = r0;
            for (int k = r0; k < r1; ++k) {
                const double v = run_weight(k);
                if (v > 0.0) {
                    some = k;
                    at_last = sum;
                    if (run < 0 && sum + v > target) {
                        run = k;
                        at_run = sum;
                    }
                }
                sum += v;
            }
            double before = lane_value(run < 0 ? at_last : at_run, who);
            run = lane_value(run < 0 ? some : run, who);
            const int64_t n0 = run * a.run, n1 = n0 + a.run < a.N ? n0 + a.run : a.N;
            int last = -1;
            for (int64_t at = n0; at < n1 && next < 0; at += RUN) {
                double ep[8], eq[8], mine = 0.0;
                drawn.eight(at + 8 * lane, n1, rest, ep, eq);
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    ep[e] = weight(ep[e], eq[e]);
                    mine += ep[e];
                }
                const double scan = sum_scan(mine);
                const int who = crossing(before + scan, mine, target);
                if (who >= 0) {
                    double upto = before + (scan - mine);
                    int pick = -1, some = -1;
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        upto += ep[e];
                        if (ep[e] > 0.0) some = e;
                        if (pick < 0 && ep[e] > 0.0 && upto > target) pick = e;
                    }
                    const int word = lane_value(pick < 0 ? some : pick, who);
                    last = int(at + 8 * who + word);
                    if (lane_value(before + scan, who) > target) next = last;
                }
                before += lane_value(scan, 63);
            }
            if (next < 0) next = last;  // (roundings: the last word with a weight)
        }
    }
    for (int i = lane; i <= a.L; i += 64)
        a.out[b * (a.L + 1) + i] = i < d.count ? a.tokens[b * a.L + i] : (i == d.count ? next : -1);
    if (lane == 0) a.count[b] = d.count;
}

// ---------------------------------------------------------------------------
// Host side.
// ---------------------------------------------------------------------------
struct DLayout {
    int rows, runs, parts, vectors;  // vectors: of a turn, a thread
    int64_t turn, turns, per, blocks, pieces, run;
    size_t part, rest, dec, total;
};

DLayout draft_layout(int64_t B, int64_t L, int64_t N, bool draft)
{
    DLayout l{};
    l.rows = int(L + 1 + (draft ? L : 0));
    // Turns of four vectors a thread, of two where that leaves compute units idle, in as
    // many equal shares as blocks run together: a block's start and joins cost it half a turn.
    const int64_t all_rows = std::max<int64_t>(B * l.rows, 1);
    l.vectors = all_rows * ((N + 4 * VSTEP - 1) / (4 * VSTEP)) < 512 ? 2 : 4;
    l.turn = l.vectors * VSTEP;
    l.turns = (N + l.turn - 1) / l.turn;
    l.per = (all_rows * l.turns + MOST_TURNS - 1) / MOST_TURNS;
    l.blocks = (all_rows * l.turns + l.per - 1) / l.per;
    l.pieces = (l.turns + l.per - 1) / l.per + 1;
    l.run = ((N + RUN - 1) / RUN + MAX_RUNS - 1) / MAX_RUNS * RUN;
    l.runs = int((N + l.run - 1) / l.run);
    // blocks of a row's runs: a wave one run, or as many as leaves three blocks a compute unit
    const int64_t most = (l.runs + DT / 64 - 1) / (DT / 64);
    l.parts = int(std::clamp<int64_t>(768 / std::max<int64_t>(B, 1), 1, most));
    size_t at = 0;
    auto take = [&](size_t bytes) {
        const size_t p = at;
        at += align256(bytes);
        return p;
    };
    l.part = take(size_t(B) * l.rows * l.pieces * sizeof(Piece));
    l.rest = take(size_t(B) * l.runs * sizeof(Run));
    l.dec = take(size_t(B) * sizeof(Decision));
    l.total = at;
    return l;
}

template <bool PB, bool QB>
hipError_t launch_draft(const DArgs &a, const DLayout &l, hipStream_t st)
{
    const dim3 grid{unsigned(l.blocks)};
    if (l.vectors == 2) hipLaunchKernelGGL((draft_rows_kernel<PB, QB, 2>), grid, dim3(DT), 0, st, a);
    else hipLaunchKernelGGL((draft_rows_kernel<PB, QB, 4>), grid, dim3(DT), 0, st, a);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((draft_rest_kernel<PB, QB>), dim3(unsigned(a.B * a.parts)), dim3(DT), 0, st, a);
    if ((e = hipGetLastError()) != hipSuccess) return e;
    hipLaunchKernelGGL((draft_draw_kernel<PB, QB>), dim3(unsigned(a.B)), dim3(64), 0, st, a);
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
    a.turn = l.turn;
    a.turns = l.turns;
    a.per = l.per;
    a.pieces = l.pieces;
    a.unsure = UNSURE + UNSURE_TURN * double(std::min(l.per, l.turns));
    a.run = l.run;
    a.runs = l.runs;
    a.parts = l.parts;
    a.tokens = c.tokens;
    a.lens = c.lens;
    a.u = c.u;
    a.r = c.r;
    a.temp = c.temp;
    a.count = c.count;
    a.out = c.out;
    a.err = c.err;
    a.part = reinterpret_cast<Piece *>(ws + l.part);
    a.rest = reinterpret_cast<Run *>(ws + l.rest);
    a.dec = reinterpret_cast<Decision *>(ws + l.dec);
    const bool pb = c.p_dtype == BSQ_BF16, qb = c.Q ? c.q_dtype == BSQ_BF16 : pb;
    if (pb) return qb ? launch_draft<true, true>(a, l, st) : launch_draft<true, false>(a, l, st);
    return qb ? launch_draft<false, true>(a, l, st) : launch_draft<false, false>(a, l, st);
}

}  // namespace bsq
