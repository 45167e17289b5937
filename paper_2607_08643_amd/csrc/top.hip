// The K largest logits of every row of a vocabulary with their words (descending,
// equal ones by the lower word; -inf and NaN never listed), and the log of the sum of
// exponentials over the whole row: one reading of the logits.
//
// A row is cut into segments, a block each. A wave keeps, in LDS, the words that may be
// among the K largest: those not below a bound that only rises. The bound: every lane
// knows the largest of what it has read; if in each of the W waves that hold words at
// least ceil(K / W) lanes have read one of b or more, at least K words are not below b.
// It is found from the lanes' maxima by a binary search over their bits with ballots,
// after 1, 2, 4, 8, ... chunks, and the waves read each other's without waiting. Random
// rows pass some 1.6 K words each time the words read double. A wave whose list is
// full cuts it to its K largest (exactly, by the 64-bit keys of value and word), so that
// rows in rising order or of equal values need no more room.
//
// A second launch joins a row's segments: keys not below a bound found the same way, each
// placed by the number of larger ones.
//
// Bound by memory for many rows, by the two launches' latency for few.
#include <algorithm>

#include "vocab_rows.h"

namespace bsq {
namespace {

constexpr int TT = 512;                 // threads of a block
constexpr int TW = TT / 64;             // its waves
constexpr int64_t TVEC = 8 * TT;        // words of a vector a thread
constexpr int WCAP = 512;               // keys a wave holds
constexpr int SEG_CAP = TW * WCAP;      // keys a segment leaves
constexpr int64_t MAX_SEGS = 64;        // of a row: one a lane
constexpr int64_t MAX_ITEMS = 2048;     // segments in a launch (workspace: 32 KiB each)
constexpr float LOG2E = 1.4426950408889634f;
static_assert(BSQ_MAX_TOP + 64 <= WCAP - 64, "a cut list has room for more");

struct TArgs {
    const void *Z;
    int64_t ldz, T, N, len;   // len: words of a segment
    int segs, K;
    float scale;
    int64_t row0;             // first row of the launch
    uint64_t *keys;           // [rows of the launch][segs][SEG_CAP]
    int32_t *counts;          // [rows of the launch][segs]
    float2 *stat;             // [rows of the launch][segs]: largest logit, sum of exponentials against it
    int32_t *ids;
    float *top, *lse;
};

// Values in order as whole numbers (-0 as +0).
__device__ __forceinline__ uint32_t ordered(float z)
{
    const uint32_t u = __float_as_uint(z + 0.0f);
    return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}
__device__ __forceinline__ float unordered(uint32_t k)
{
    return __uint_as_float((k & 0x80000000u) ? (k & 0x7fffffffu) : ~k);
}
// of equal values the lower word has the larger key; no key is 0
__device__ __forceinline__ uint64_t key_of(float z, uint32_t word) { return (uint64_t(ordered(z)) << 32) | ~word; }

constexpr uint32_t LOWEST = 0x00800000u;  // ordered(the lowest finite value)

__device__ __forceinline__ int lanes_below(uint64_t mask)
{
    return __builtin_amdgcn_mbcnt_hi(uint32_t(mask >> 32), __builtin_amdgcn_mbcnt_lo(uint32_t(mask), 0));
}

// LDS written by some lanes of a wave and read by others: in program order.
__device__ __forceinline__ void wave_sync()
{
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

// The q-th largest of the lanes' values (0 where there are fewer above LOWEST).
__device__ __forceinline__ uint32_t lanes_rank(uint32_t v, int q)
{
    uint32_t at = 0;
    for (int bit = 31; bit >= 0; --bit) {
        const uint32_t up = at | (1u << bit);
        if (__popcll(__ballot(v >= up)) >= q) at = up;
    }
    return at < LOWEST ? 0u : at;
}

// The K largest of the n (<= 512, >= K) keys of a wave's list, in no order; the
// smallest of them is returned.
__device__ __forceinline__ uint64_t wave_cut(uint64_t *list, int n, int K)
{
    const int lane = threadIdx.x & 63;
    uint64_t k[WCAP / 64];
#pragma unroll
    for (int i = 0; i < WCAP / 64; ++i) k[i] = 64 * i + lane < n ? list[64 * i + lane] : 0;
    uint64_t at = 0;
    for (int bit = 63; bit >= 0; --bit) {
        const uint64_t up = at | (uint64_t(1) << bit);
        int c = 0;
#pragma unroll
        for (int i = 0; i < WCAP / 64; ++i) c += __popcll(__ballot(k[i] >= up));
        if (c >= K) at = up;
    }
    wave_sync();
    int pos = 0;
#pragma unroll
    for (int i = 0; i < WCAP / 64; ++i) {
        const uint64_t keep = __ballot(k[i] >= at);
        if (k[i] >= at) list[pos + lanes_below(keep)] = k[i];
        pos += __popcll(keep);
    }
    wave_sync();
    return at;
}

__device__ __forceinline__ float finite_ref(float m) { return m == -__builtin_inff() ? 0.0f : m; }

// Largest value and sum of exponentials against it, joined with another pair.
__device__ __forceinline__ void join(float &m, float &s, float m2, float s2, float c)
{
    const float mm = m2 > m ? m2 : m, ref = (mm == __builtin_inff()) ? 0.0f : finite_ref(mm);
    s = s * __builtin_amdgcn_exp2f((m - ref) * c) + s2 * __builtin_amdgcn_exp2f((m2 - ref) * c);
    m = mm;
}

constexpr int CV = 2;  // vectors of a chunk

template <bool BF16>
__global__ __launch_bounds__(TT) void top_rows_kernel(const TArgs a)
{
    __shared__ uint64_t s_list[TW][WCAP];
    __shared__ uint32_t s_bound[TW];
    __shared__ int s_count[TW];
    __shared__ float2 s_stat[TW];
    const int t = threadIdx.x, lane = t & 63;
    const int w = __builtin_amdgcn_readfirstlane(t >> 6);
    const int64_t r = blockIdx.x / a.segs;
    const int seg = int(blockIdx.x - r * a.segs);
    const int64_t row = a.row0 + r;
    const int64_t n0 = seg * a.len, n1 = n0 + a.len < a.N ? n0 + a.len : a.N;
    const void *z = BF16 ? static_cast<const void *>(static_cast<const uint16_t *>(a.Z) + row * a.ldz)
                         : static_cast<const float *>(a.Z) + row * a.ldz;
    const float c = a.scale * LOG2E;
    // waves that hold words, and how many lanes of each the bound asks for
    const int64_t full = (n1 - n0 + 511) / 512;
    const int waves = full < TW ? int(full) : TW, q = (a.K + waves - 1) / waves;

    float m = -__builtin_inff(), s = 0.0f;
    uint64_t floor_key = 0; // of the wave's list, once it was cut
    int held = 0;
    float thr = unordered(LOWEST);
    uint64_t *list = s_list[w];

    Words8<BF16> next[CV];
    auto load = [&](int64_t base) {
#pragma unroll
        for (int k = 0; k < CV; ++k) {
            const int64_t at = base + k * TVEC + 8 * t;
            next[k].load(z, at < n1 ? at : n1, n1);
        }
    };
    load(n0);
    int chunk = 0;
    for (int64_t base = n0; base < n1; base += CV * TVEC, ++chunk) {
        Words8<BF16> cur[CV];
#pragma unroll
        for (int k = 0; k < CV; ++k) cur[k] = next[k];
        if (base + CV * TVEC < n1) load(base + CV * TVEC);
        float mx = -__builtin_inff();
#pragma unroll
        for (int k = 0; k < CV; ++k)
#pragma unroll
            for (int e = 0; e < 8; ++e) mx = fmaxf(mx, cur[k][e]);
        // the sum, against the largest that the thread has read
        const float mm = mx > m ? mx : m, ref = (mm == __builtin_inff()) ? 0.0f : finite_ref(mm);
        if (mx > m) {
            s *= __builtin_amdgcn_exp2f((m - ref) * c);
            m = mx;
        }
#pragma unroll
        for (int k = 0; k < CV; ++k)
#pragma unroll
            for (int e = 0; e < 8; ++e) s += __builtin_amdgcn_exp2f((cur[k][e] - ref) * c);
        // the bound
        if ((chunk & (chunk + 1)) == 0) {
            const uint32_t b = q <= 64 ? lanes_rank(ordered(m), q) : 0u;
            if (lane == 0) s_bound[w] = b;
            if (chunk == 0) __syncthreads();
        }
        uint32_t bound = ~0u;
#pragma unroll
        for (int k = 0; k < TW; ++k) {
            const uint32_t b = reinterpret_cast<volatile uint32_t *>(s_bound)[k];
            if (k < waves && b < bound) bound = b;
        }
        if (bound > LOWEST) {
            const float f = unordered(bound);
            thr = f > thr ? f : thr;
        }
        if (__ballot(mx >= thr) == 0) continue;
        uint32_t pass = 0;
#pragma unroll
        for (int k = 0; k < CV; ++k)
#pragma unroll
            for (int e = 0; e < 8; ++e) pass |= (cur[k][e] >= thr) ? 1u << (8 * k + e) : 0u;
        while (__ballot(pass != 0)) {
            const int e = pass ? __builtin_ctz(pass) : 0;
            float v = cur[0][0];
#pragma unroll
            for (int k = 0; k < CV; ++k)
#pragma unroll
                for (int i = 0; i < 8; ++i) v = (e == 8 * k + i) ? cur[k][i] : v;
            const uint64_t key = key_of(v, uint32_t(base + (e >> 3) * TVEC + 8 * t + (e & 7)));
            const bool put = pass != 0 && key > floor_key;
            pass &= pass - 1;
            const uint64_t mask = __ballot(put);
            if (put) list[held + lanes_below(mask)] = key;
            held += __popcll(mask);
            if (held > WCAP - 64) {
                wave_sync();
                floor_key = wave_cut(list, held, a.K);
                held = a.K;
                const float f = unordered(uint32_t(floor_key >> 32));
                thr = f > thr ? f : thr;
            }
        }
    }
    // what is left at the bound of the whole segment, and its largest and sum
    {
        const uint32_t b = q <= 64 ? lanes_rank(ordered(m), q) : 0u;
        if (lane == 0) s_bound[w] = b;
    }
    for (int d = 32; d > 0; d >>= 1) join(m, s, __shfl_xor(m, d), __shfl_xor(s, d), c);
    wave_sync();
    __syncthreads();
    uint32_t bound = ~0u;
#pragma unroll
    for (int k = 0; k < TW; ++k)
        if (k < waves && s_bound[k] < bound) bound = s_bound[k];
    int kept = 0;
    for (int i = 0; i < held; i += 64) {
        const uint64_t key = i + lane < held ? list[i + lane] : 0;
        kept += __popcll(__ballot(key != 0 && uint32_t(key >> 32) >= bound));
    }
    if (lane == 0) {
        s_count[w] = kept;
        s_stat[w] = make_float2(m, s);
    }
    __syncthreads();
    int at = 0, all = 0;
    for (int k = 0; k < TW; ++k) {
        at += k < w ? s_count[k] : 0;
        all += s_count[k];
    }
    const int64_t item = blockIdx.x;
    uint64_t *out = a.keys + item * SEG_CAP + at;
    for (int i = 0; i < held; i += 64) {
        const uint64_t key = i + lane < held ? list[i + lane] : 0;
        const bool keep = key != 0 && uint32_t(key >> 32) >= bound;
        const uint64_t mask = __ballot(keep);
        if (keep) out[lanes_below(mask)] = key;
        out += __popcll(mask);
    }
    if (t == 0) {
        for (int k = 1; k < TW; ++k) join(m, s, s_stat[k].x, s_stat[k].y, c);
        a.counts[item] = all;
        a.stat[item] = make_float2(m, s);
    }
}

// ---------------------------------------------------------------------------
// A row's segments joined. Keys go through LDS in batches; each batch is cut to
// the K largest, sorted.
// ---------------------------------------------------------------------------
constexpr int JCAP = 4096;

// s_keys[0 .. n) -> its min(n, K) largest in order, at the front; returns their number.
// s_rank: room for as many. By the whole block, ends with a barrier.
__device__ __forceinline__ int block_cut(uint64_t *s_keys, uint64_t *s_rank, int n, int K, uint32_t *s_bound, int *s_n)
{
    const int t = threadIdx.x, lane = t & 63, w = t >> 6;
    const int keep = n < K ? n : K;
    // a bound that at least K keys reach, as in the first launch
    const int q = (K + TW - 1) / TW;
    uint64_t own[JCAP / TT];
    uint32_t best = 0;
#pragma unroll
    for (int i = 0; i < JCAP / TT; ++i) {
        own[i] = i * TT + t < n ? s_keys[i * TT + t] : 0;
        const uint32_t v = uint32_t(own[i] >> 32);
        best = v > best ? v : best;
    }
    const uint32_t b = lanes_rank(best, q);
    if (lane == 0) s_bound[w] = b;
    if (t == 0) *s_n = 0;
    __syncthreads();
    uint32_t bound = ~0u;
#pragma unroll
    for (int k = 0; k < TW; ++k) bound = s_bound[k] < bound ? s_bound[k] : bound;
#pragma unroll
    for (int i = 0; i < JCAP / TT; ++i) {
        const bool in = own[i] != 0 && uint32_t(own[i] >> 32) >= bound;
        const uint64_t mask = __ballot(in);
        int at = 0;
        if (lane == 0 && mask) at = atomicAdd(s_n, __popcll(mask));
        at = __shfl(at, 0);
        if (in) s_rank[at + lanes_below(mask)] = own[i];
    }
    __syncthreads();
    const int m = *s_n;
    // every key's place is the number of larger ones (no two are equal)
    for (int i = t; i < m; i += TT) {
        const uint64_t key = s_rank[i];
        int place = 0;
        for (int k = 0; k < m; ++k) place += s_rank[k] > key ? 1 : 0;
        if (place < keep) s_keys[place] = key;
    }
    __syncthreads();
    return keep;
}

__global__ __launch_bounds__(TT) void top_join_kernel(const TArgs a)
{
    __shared__ uint64_t s_keys[JCAP], s_rank[JCAP];
    __shared__ uint32_t s_bound[TW];
    __shared__ int s_n, s_off[MAX_SEGS + 1];
    const int t = threadIdx.x, lane = t & 63;
    const int64_t r = blockIdx.x, row = a.row0 + r;
    if (t < 64) {
        int end = lane < a.segs ? a.counts[r * a.segs + lane] : 0;
        for (int d = 1; d < 64; d <<= 1) {
            const int o = __shfl_up(end, d);
            if (lane >= d) end += o;
        }
        s_off[lane + 1] = end;
        if (lane == 0) s_off[0] = 0;
    }
    __syncthreads();
    const int all = s_off[a.segs];
    int n = 0;
    for (int done = 0; done < all;) {
        if (n == JCAP) {
            __syncthreads();
            n = block_cut(s_keys, s_rank, n, a.K, s_bound, &s_n);
        }
        const int take = all - done < JCAP - n ? all - done : JCAP - n;
        for (int i = t; i < take; i += TT) {
            int g = 0;  // the segment of key done + i
#pragma unroll
            for (int h = 32; h > 0; h >>= 1)
                if (g + h < a.segs && s_off[g + h] <= done + i) g += h;
            s_keys[n + i] = a.keys[(r * a.segs + g) * SEG_CAP + (done + i - s_off[g])];
        }
        n += take;
        done += take;
    }
    __syncthreads();
    n = block_cut(s_keys, s_rank, n, a.K, s_bound, &s_n);
    for (int i = t; i < a.K; i += TT) {
        const uint64_t key = i < n ? s_keys[i] : 0;
        a.ids[row * a.K + i] = i < n ? int32_t(~uint32_t(key)) : -1;
        a.top[row * a.K + i] = i < n ? unordered(uint32_t(key >> 32)) : -__builtin_inff();
    }
    if (a.lse && t < 64) {
        const float c = a.scale * LOG2E;
        const float2 v = lane < a.segs ? a.stat[r * a.segs + lane] : make_float2(-__builtin_inff(), 0.0f);
        float m = v.x, s = v.y;
        for (int d = 32; d > 0; d >>= 1) join(m, s, __shfl_xor(m, d), __shfl_xor(s, d), c);
        // (a row with +inf: its sum is against 0)
        if (t == 0) a.lse[row] = (m == __builtin_inff() ? 0.0f : m * a.scale) + logf(s);
    }
}

// ---------------------------------------------------------------------------
// Host side.
// ---------------------------------------------------------------------------
struct TLayout {
    int segs;
    int64_t len, rows;  // words of a segment, rows of a launch
    size_t keys, counts, stat, total;
};

TLayout top_layout(int64_t T, int64_t N)
{
    TLayout l{};
    // segments until the launch fills the compute units (four blocks each)
    const int64_t unit = CV * TVEC, steps = (N + unit - 1) / unit;
    const int64_t want = std::clamp<int64_t>(MAX_ITEMS / std::max<int64_t>(T, 1), 1, std::min(MAX_SEGS, steps));
    l.len = (steps + want - 1) / want * unit;
    l.segs = int((N + l.len - 1) / l.len);
    l.rows = std::min<int64_t>(std::max<int64_t>(T, 1), MAX_ITEMS / l.segs);
    size_t at = 0;
    auto take = [&](size_t bytes) {
        const size_t p = at;
        at += align256(bytes);
        return p;
    };
    l.keys = take(size_t(l.rows) * l.segs * SEG_CAP * 8);
    l.counts = take(size_t(l.rows) * l.segs * 4);
    l.stat = take(size_t(l.rows) * l.segs * 8);
    l.total = at;
    return l;
}

}  // namespace

size_t top_ws_bytes(int64_t T, int64_t N) { return top_layout(T, N).total; }

hipError_t launch_top_logits(const TopCall &c, hipStream_t st)
{
    const TLayout l = top_layout(c.T, c.N);
    char *ws = static_cast<char *>(c.ws);
    TArgs a{};
    a.Z = c.Z;
    a.ldz = c.ldz;
    a.T = c.T;
    a.N = c.N;
    a.len = l.len;
    a.segs = l.segs;
    a.K = c.K;
    a.scale = c.scale;
    a.keys = reinterpret_cast<uint64_t *>(ws + l.keys);
    a.counts = reinterpret_cast<int32_t *>(ws + l.counts);
    a.stat = reinterpret_cast<float2 *>(ws + l.stat);
    a.ids = c.ids;
    a.top = c.top;
    a.lse = c.lse;
    hipError_t e = hipSuccess;
    for (int64_t r0 = 0; e == hipSuccess && r0 < c.T; r0 += l.rows) {
        const int64_t rows = std::min(l.rows, c.T - r0);
        a.row0 = r0;
        const dim3 grid(unsigned(rows * l.segs));
        if (c.z_dtype == BSQ_BF16) hipLaunchKernelGGL((top_rows_kernel<true>), grid, dim3(TT), 0, st, a);
        else hipLaunchKernelGGL((top_rows_kernel<false>), grid, dim3(TT), 0, st, a);
        if ((e = hipGetLastError()) != hipSuccess) break;
        hipLaunchKernelGGL(top_join_kernel, dim3(unsigned(rows)), dim3(TT), 0, st, a);
        e = hipGetLastError();
    }
    return e;
}

}  // namespace bsq
