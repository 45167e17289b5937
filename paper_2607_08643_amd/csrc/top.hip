// The K largest logits of every row of a vocabulary with their words (descending,
// equal ones by the lower word; -inf and NaN never listed), and the log of the sum of
// exponentials over the whole row: one reading of the logits.
//
// A block reads a row, or a segment of it where there are few rows. A wave keeps, in LDS,
// the words that may be among the K largest: those not below a bound that only rises. The bound: every lane
// knows the largest of what it has read; if in each of the W waves that hold words at
// least ceil(K / W) lanes have read one of b or more, at least K words are not below b.
// It is found from the lanes' maxima by a binary search over their bits with ballots,
// after 1, 2, 4, 8, ... chunks, and the waves read each other's without waiting. Random
// rows pass some 1.6 K words each time the words read double. A wave whose list is
// full cuts it to its K largest (exactly, by the 64-bit keys of value and word), so that
// rows in rising order or of equal values need no more room.
//
// What is left is cut to a bound found the same way; each key's place is the number of
// larger ones. Where rows are cut into segments a second launch does that for all
// segments of a row.
//
// 512 rows of 151936 words in bf16, K = 64: 42 us (156 MB, 3.7 TB/s). With parts left
// out of a run of 44: reading and the bound alone 26, all but the exponentials 38, all but
// the last cut 39, without words that pass (and so nothing to cut) 33. Few rows take two
// launches of 7 to 8 us, chains of a few dependent steps.
#include <algorithm>
#include <type_traits>

#include "vocab_rows.h"

namespace bsq {
namespace {

constexpr int TT = 1024;                // threads of a block
constexpr int TW = TT / 64;             // its waves
constexpr int64_t TVEC = 8 * TT;        // words of a vector a thread
constexpr int WCAP = 384;               // keys a wave holds
constexpr int OWN = WCAP / 64;          // a lane
constexpr int LIST = TW * WCAP;         // a block
constexpr int PASSED = 16;              // lanes whose words a wave looks through in LDS
constexpr int BINS = 256;               // of values, four a lane
constexpr int FEW = 1024;               // keys that are put in order by counting
constexpr int64_t MAX_SEGS = 64;        // of a row: one a lane
constexpr int64_t MAX_ITEMS = 256;      // segments in a launch, where rows are cut (workspace: 48 KiB each)
constexpr float LOG2E = 1.4426950408889634f;
static_assert(BSQ_MAX_TOP + 64 <= WCAP - 64, "a cut list has room for more");
static_assert(LIST < 65536, "places are of 16 bits");

struct TArgs {
    const void *Z;
    int64_t ldz, N, len;   // len: words of a segment
    int segs, K;
    float scale;
    int64_t row0;             // first row of the launch
    uint64_t *keys;           // [rows of the launch][segs][LIST]
    int32_t *counts;          // [rows of the launch][segs]
    float2 *stat;             // [rows of the launch][segs]: largest logit, sum of exponentials against it
    int32_t *ids;
    float *top, *lse;
};

struct TShared {
    uint64_t list[LIST];      // of the waves; then the keys that reach the bound
    uint32_t place[LIST / 2]; // of these: the number of larger ones, two of 16 bits
    uint64_t best[BSQ_MAX_TOP];
    __attribute__((aligned(16))) uint32_t bound[TW];
    __attribute__((aligned(16))) uint32_t bins[BINS];
    uint32_t low[TW];         // before a cut: the waves' smallest key, its value; their largest in stat; bins of 0
    int count[2][TW];
    float2 stat[TW];          // of the waves
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

// The q-th largest of the lanes' values, cut to its upper 16 bits: a bound that may lie a
// little below (0 where there are fewer above LOWEST).
__device__ __forceinline__ uint32_t lanes_rank(uint32_t v, int q)
{
    uint32_t at = 0;
#pragma unroll
    for (int bit = 31; bit >= 16; --bit) {
        const uint32_t up = at | (1u << bit);
        if (__popcll(__ballot(v >= up)) >= q) at = up;
    }
    return at < LOWEST ? 0u : at;
}

// The K largest of the n (<= WCAP, >= K) keys of a wave's list, in no order; the
// smallest of them is returned.
__device__ __forceinline__ uint64_t wave_cut(uint64_t *list, int n, int K)
{
    const int lane = threadIdx.x & 63;
    uint64_t k[OWN];
#pragma unroll
    for (int i = 0; i < OWN; ++i) k[i] = 64 * i + lane < n ? list[64 * i + lane] : 0;
    uint64_t at = 0;
    for (int bit = 63; bit >= 0; --bit) {
        const uint64_t up = at | (uint64_t(1) << bit);
        int c = 0;
#pragma unroll
        for (int i = 0; i < OWN; ++i) c += __popcll(__ballot(k[i] >= up));
        if (c >= K) at = up;
    }
    wave_sync();
    int pos = 0;
#pragma unroll
    for (int i = 0; i < OWN; ++i) {
        const uint64_t keep = __ballot(k[i] >= at);
        if (k[i] >= at) list[pos + lanes_below(keep)] = k[i];
        pos += __popcll(keep);
    }
    wave_sync();
    return at;
}

__device__ __forceinline__ float finite_ref(float m) { return m == -__builtin_inff() ? 0.0f : m; }

// The lanes' largest values and sums of exponentials against them, joined. (Sums beside
// an infinite largest value are against 0.)
__device__ __forceinline__ void wave_join(float &m, float &s, float c)
{
    const float mm = wave_max(m), ref = (mm == __builtin_inff()) ? 0.0f : finite_ref(mm);
    s = wave_sum(s * __builtin_amdgcn_exp2f((m - ref) * c));
    m = mm;
}

// The smallest of the waves' bounds (those without words leave the largest).
__device__ __forceinline__ uint32_t block_bound(const uint32_t *s_bound)
{
    uint32_t bound = ~0u;
#pragma unroll
    for (int h = 0; h < TW; h += 4) {
        const vr_u32x4_t b = *reinterpret_cast<const volatile vr_u32x4_t *>(s_bound + h);
#pragma unroll
        for (int k = 0; k < 4; ++k) bound = b[k] < bound ? b[k] : bound;
    }
    return bound;
}

// A wave's bound: what q lanes reach.
__device__ __forceinline__ uint32_t wave_bound(uint32_t best, int q, bool words)
{
    return !words ? ~0u : (q <= 64 ? lanes_rank(best, q) : 0u);
}

// Of the lanes' keys (0: none) those of `least` or more: a wave's masks, and their number
// before the wave's and of all waves. (A barrier; calls take turns with `slot`.)
__device__ __forceinline__ void count_keys(const uint64_t (&own)[OWN], uint64_t least, uint64_t (&mask)[OWN], int &before,
                                           int &all, int slot, TShared &sh)
{
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    int count = 0;
#pragma unroll
    for (int i = 0; i < OWN; ++i) {
        mask[i] = __ballot(own[i] != 0 && own[i] >= least);
        count += __popcll(mask[i]);
    }
    if (lane == 0) sh.count[slot][w] = count;
    __syncthreads();
    before = 0;
    all = 0;
#pragma unroll
    for (int k = 0; k < TW; ++k) {
        const int n = sh.count[slot][k];
        before += k < w ? n : 0;
        all += n;
    }
}

__device__ __forceinline__ void put_keys(const uint64_t (&own)[OWN], const uint64_t (&mask)[OWN], uint64_t *out)
{
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int i = 0; i < OWN; ++i) {
        if ((mask[i] >> lane) & 1) out[lanes_below(mask[i])] = own[i];
        out += __popcll(mask[i]);
    }
}

// Before a cut and a barrier: what it needs to know of the wave's keys.
__device__ __forceinline__ void prepare_cut(const uint64_t (&own)[OWN], TShared &sh)
{
    const int t = threadIdx.x;
    uint32_t low = ~0u;
#pragma unroll
    for (int i = 0; i < OWN; ++i) {
        const uint32_t v = own[i] != 0 ? uint32_t(own[i] >> 32) : ~0u;
        low = v < low ? v : low;
    }
    low = lane_value(wave_scan(low, ~0u, [](uint32_t x, uint32_t y) { return x < y ? x : y; }), 63);
    if ((t & 63) == 0) sh.low[t >> 6] = low;
    if (t < BINS) sh.bins[t] = 0;
}

// A bound nearer to the K-th largest: the values from `bound` (or the smallest) to the largest
// in 256 bins, the lowest bin that the K largest reach. (A barrier.)
__device__ __forceinline__ uint32_t bin_bound(const uint64_t (&own)[OWN], uint32_t bound, int K, TShared &sh)
{
    const int lane = threadIdx.x & 63;
    float most = -__builtin_inff();
    uint32_t low = ~0u;
#pragma unroll
    for (int k = 0; k < TW; ++k) {
        most = fmaxf(most, sh.stat[k].x);
        low = sh.low[k] < low ? sh.low[k] : low;
    }
    bound = low > bound ? low : bound;
    const uint32_t last = ordered(most), range = last > bound ? last - bound : 0;
    const int shift = range < BINS ? 0 : 24 - __builtin_clz(range);
#pragma unroll
    for (int i = 0; i < OWN; ++i) {
        const uint32_t v = uint32_t(own[i] >> 32);
        if (own[i] != 0 && v >= bound) atomicAdd(&sh.bins[(v - bound) >> shift], 1u);
    }
    __syncthreads();
    // lane 0 has the upper four bins
    const int first = BINS - 4 - 4 * lane;
    const vr_u32x4_t n = *reinterpret_cast<const vr_u32x4_t *>(sh.bins + first);
    const int own_n = int(n[0] + n[1] + n[2] + n[3]);
    const int upto = wave_scan(own_n, 0, [](int x, int y) { return x + y; });
    const uint64_t reach = __ballot(upto >= K);
    if (reach == 0) return bound;
    int bin = 0, sum = upto - own_n;
#pragma unroll
    for (int k = 3; k >= 0; --k) {
        if (sum < K) bin = first + k;
        sum += int(n[k]);
    }
    bin = lane_value(bin, __builtin_ctzll(reach));
    return bound + (uint32_t(bin) << shift);
}

// The K largest of the block's keys in order into sh.best; returns their number. No two
// keys are equal; at least min(K, all) are not below `bound`. (sh.list is written: every wave
// has read its own. Ends with a barrier.)
__device__ __forceinline__ int block_cut(const uint64_t (&own)[OWN], uint32_t bound, int K, TShared &sh)
{
    const int t = threadIdx.x, lane = t & 63, w = __builtin_amdgcn_readfirstlane(t >> 6);
    uint64_t least = uint64_t(bin_bound(own, bound, K, sh)) << 32, mask[OWN];
    int before, m;
    count_keys(own, least, mask, before, m, 0, sh);
    if (m > FEW) {
        // many equal values: the K-th largest key, bit by bit
        least = 0;
        int slot = 1;
        for (int bit = 63; bit >= 0; --bit) {
            const uint64_t up = least | (uint64_t(1) << bit);
            int n;
            count_keys(own, up, mask, before, n, slot, sh);
            slot ^= 1;
            if (n >= K) least = up;
        }
        count_keys(own, least, mask, before, m, slot, sh);
    }
    put_keys(own, mask, sh.list + before);
    for (int i = t; 2 * i < m; i += TT) sh.place[i] = 0;
    __syncthreads();
    // a wave compares its share of the keys with all, four a lane (one reading of LDS for
    // four comparisons)
    const int k0 = m * w / TW, k1 = m * (w + 1) / TW;
    for (int i0 = 0; i0 < m; i0 += 256) {
        uint64_t key[4];
        uint32_t place[4] = {0u, 0u, 0u, 0u};
#pragma unroll
        for (int e = 0; e < 4; ++e) key[e] = i0 + 64 * e + lane < m ? sh.list[i0 + 64 * e + lane] : ~uint64_t(0);
#pragma unroll 4
        for (int k = k0; k < k1; ++k) {
            const uint64_t other = sh.list[k];
#pragma unroll
            for (int e = 0; e < 4; ++e) place[e] += other > key[e] ? 1u : 0u;
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int i = i0 + 64 * e + lane;
            if (i < m) atomicAdd(&sh.place[i >> 1], place[e] << (16 * (i & 1)));
        }
    }
    __syncthreads();
    const int keep = m < K ? m : K;
    for (int i = t; i < m; i += TT) {
        const int at = (sh.place[i >> 1] >> (16 * (i & 1))) & 0xffff;
        if (at < keep) sh.best[at] = sh.list[i];
    }
    __syncthreads();
    return keep;
}

__device__ __forceinline__ void write_row(const TArgs &a, int64_t row, int n, const TShared &sh)
{
    for (int i = threadIdx.x; i < a.K; i += TT) {
        const uint64_t key = i < n ? sh.best[i] : 0;
        a.ids[row * a.K + i] = i < n ? int32_t(~uint32_t(key)) : -1;
        a.top[row * a.K + i] = i < n ? unordered(uint32_t(key >> 32)) : -__builtin_inff();
    }
}

// (a row with +inf: its sum is against 0)
__device__ __forceinline__ float row_lse(const TArgs &a, float m, float s)
{
    return (m == __builtin_inff() ? 0.0f : m * a.scale) + logf(s);
}

// WHOLE: a block a row, its results; else a segment's candidates, largest logit and sum.
// 32 bytes a thread and turn; eight waves a SIMD hide their latency (64 registers).
template <bool BF16, bool WHOLE>
__global__ __launch_bounds__(TT) __attribute__((amdgpu_waves_per_eu(8, 8))) void top_rows_kernel(const TArgs a)
{
    constexpr int CV = BF16 ? 2 : 1;                // vectors of a chunk
    constexpr int E = 8 * CV, AT_ONCE = 64 / E;     // words of a lane; lanes whose words a wave looks through at once
    using Raw = std::conditional_t<BF16, uint16_t, uint32_t>;
    __shared__ TShared sh;
    __shared__ __attribute__((aligned(16))) Raw s_raw[TW][PASSED][E];
    __shared__ int s_from[TW][PASSED];
    const int t = threadIdx.x, lane = t & 63;
    const int w = __builtin_amdgcn_readfirstlane(t >> 6);
    const int64_t r = WHOLE ? blockIdx.x : blockIdx.x / a.segs;
    const int seg = WHOLE ? 0 : int(blockIdx.x - r * a.segs);
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
    uint64_t *list = sh.list + w * WCAP;

    Words8<BF16> next[CV];  // the next chunk's, in flight
    auto load = [&](int64_t base) {
        // (offsets of 32 bits from the chunk's first word)
        const void *p = BF16 ? static_cast<const void *>(static_cast<const uint16_t *>(z) + base)
                             : static_cast<const float *>(z) + base;
        const int64_t left = n1 - base;
        if (left >= CV * TVEC) {
#pragma unroll
            for (int k = 0; k < CV; ++k) next[k].load(p, k * unsigned(TVEC) + 8u * t);
        } else {
            const int end = int(left);
#pragma unroll
            for (int k = 0; k < CV; ++k) {
                const int at = k * int(TVEC) + 8 * t;
                next[k].load(p, at < end ? at : end, end);
            }
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
        // (taken apart again for the sum: kept, the words would take twice the registers)
#pragma unroll
        for (int k = 0; k < CV; ++k) asm volatile("" : "+v"(cur[k].raw[0]));
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
            const uint32_t b = wave_bound(ordered(m), q, w < waves);
            if (lane == 0) sh.bound[w] = b;
            if (chunk == 0) __syncthreads();
        }
        const uint32_t bound = block_bound(sh.bound);
        if (bound > LOWEST) {
            const float f = unordered(bound);
            thr = f > thr ? f : thr;
        }
        // lanes that hold a word not below it leave theirs in LDS, where the wave looks through them
        for (uint64_t some = __ballot(mx >= thr); some != 0;) {
            const bool in = (some >> lane) & 1;
            const int rank = lanes_below(some), n = __popcll(some) < PASSED ? __popcll(some) : PASSED;
            if (in && rank < PASSED) {
                constexpr int QUADS = int(sizeof(cur[0].raw) / 16);
#pragma unroll
                for (int k = 0; k < CV; ++k)
#pragma unroll
                    for (int h = 0; h < QUADS; ++h)
                        reinterpret_cast<vr_u32x4_t *>(s_raw[w][rank])[k * QUADS + h] = cur[k].raw[h];
                s_from[w][rank] = lane;
            }
            some = __ballot(in && rank >= PASSED);
            wave_sync();
            for (int j = 0; j < n; j += AT_ONCE) {
                const int from = j + lane / E, e = lane % E;
                const bool there = from < n;
                const Raw raw = s_raw[w][there ? from : 0][e];
                const float v = BF16 ? bf16_to_f32(uint16_t(raw)) : __uint_as_float(raw);
                const uint32_t word = uint32_t(base) + (e >> 3) * unsigned(TVEC) + 8u * (64 * w + s_from[w][there ? from : 0]) + (e & 7);
                const uint64_t key = key_of(v, word);
                const bool put = there && v >= thr && key > floor_key;
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
            wave_sync();
        }
    }
    // what is left at the bound of all words, and their largest and sum
    if (chunk > 1) {
        const uint32_t b = wave_bound(ordered(m), q, w < waves);
        if (lane == 0) sh.bound[w] = b;
    }
    wave_join(m, s, c);
    if (lane == 0) sh.stat[w] = make_float2(m, s);
    uint64_t own[OWN];
#pragma unroll
    for (int i = 0; i < OWN; ++i) own[i] = 64 * i + lane < held ? list[64 * i + lane] : 0;
    if constexpr (WHOLE) prepare_cut(own, sh);
    __syncthreads();
    const uint32_t bound = block_bound(sh.bound);
    if (w == 0) {
        m = lane < TW ? sh.stat[lane].x : -__builtin_inff();
        s = lane < TW ? sh.stat[lane].y : 0.0f;
        wave_join(m, s, c);
    }
    if constexpr (WHOLE) {
        if (t == 0 && a.lse) a.lse[row] = row_lse(a, m, s);
        write_row(a, row, block_cut(own, bound, a.K, sh), sh);
    } else {
        uint64_t mask[OWN];
        int before, all;
        count_keys(own, uint64_t(bound) << 32, mask, before, all, 0, sh);
        const int64_t item = blockIdx.x;
        put_keys(own, mask, a.keys + item * LIST + before);
        if (t == 0) {
            a.counts[item] = all;
            a.stat[item] = make_float2(m, s);
        }
    }
}

// A row's segments joined, in batches of as many keys as a block holds.
__global__ __launch_bounds__(TT) void top_join_kernel(const TArgs a)
{
    __shared__ TShared sh;
    __shared__ int s_off[MAX_SEGS + 1];
    const int t = threadIdx.x, lane = t & 63, w = t >> 6;
    const int64_t r = blockIdx.x, row = a.row0 + r;
    if (t < 64) {
        const int count = lane < a.segs ? a.counts[r * a.segs + lane] : 0;
        s_off[lane + 1] = wave_scan(count, 0, [](int x, int y) { return x + y; });
        if (lane == 0) s_off[0] = 0;
    }
    if (t >= 64 && t < 128 && a.lse) {
        const float c = a.scale * LOG2E;
        const float2 v = lane < a.segs ? a.stat[r * a.segs + lane] : make_float2(-__builtin_inff(), 0.0f);
        float m = v.x, s = v.y;
        wave_join(m, s, c);
        if (lane == 0) a.lse[row] = row_lse(a, m, s);
    }
    __syncthreads();
    const int all = s_off[a.segs];
    int n = 0;
    for (int done = 0; done < all || done == 0;) {
        // what is kept, then as many more: a wave a segment
        if (t < n) sh.list[t] = sh.best[t];
        const int take = LIST - n;
        for (int g = w; g < a.segs; g += TW) {
            const int first = s_off[g], count = s_off[g + 1] - first;
            const uint64_t *src = a.keys + (r * a.segs + g) * LIST;
            for (int i0 = 0; i0 < count; i0 += WCAP) {
                uint64_t v[OWN];
#pragma unroll
                for (int e = 0; e < OWN; ++e) v[e] = i0 + 64 * e + lane < count ? src[i0 + 64 * e + lane] : 0;
#pragma unroll
                for (int e = 0; e < OWN; ++e) {
                    const int at = first + i0 + 64 * e + lane - done;
                    if (v[e] != 0 && at >= 0 && at < take) sh.list[n + at] = v[e];
                }
            }
        }
        __syncthreads();
        const int batch = n + (all - done < take ? all - done : take);
        done += take;
        uint64_t own[OWN];
        uint32_t top = 0;
#pragma unroll
        for (int i = 0; i < OWN; ++i) {
            own[i] = i * TT + t < batch ? sh.list[i * TT + t] : 0;
            const uint32_t v = uint32_t(own[i] >> 32);
            top = v > top ? v : top;
        }
        // a bound that at least K of them reach, from the waves with a key a lane, and the waves' largest
        const int full = batch / 64 < TW ? batch / 64 : TW;
        const uint32_t b = w < full || full == 0 ? wave_bound(top, full ? (a.K + full - 1) / full : 65, true) : ~0u;
        top = lane_value(wave_scan(top, 0u, [](uint32_t x, uint32_t y) { return x > y ? x : y; }), 63);
        if (lane == 0) {
            sh.bound[w] = b;
            sh.stat[w].x = top ? unordered(top) : -__builtin_inff();
        }
        prepare_cut(own, sh);
        __syncthreads();
        n = block_cut(own, block_bound(sh.bound), a.K, sh);
    }
    write_row(a, row, n, sh);
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
    // A row is cut where it is long and rows are few: into segments of 16384 words or more, up
    // to a block for every compute unit; ten segments at most while they are short (the
    // second launch costs 6 us and what they leave). Whole against cut, us, bf16, K = 64: 8
    // rows of 151936 words 22.8 against 16.1 (ten), 100 rows 23.2 against 21.4 (two), 200
    // rows 23.9 against 29.6 (two); 8 rows of 262144 words 30.9 against 17.2 (ten), 100 rows
    // 31.6 against 26.3; 8 rows of 100352 words 18.8 against 16.2 (seven), 100 rows 18.9 against
    // 19.8 (two). Up to four units, whole: 64 rows of 64000 words 14.9 against 16.1 (in fp32
    // 16.8 against 16.3), of 32003 words 13.3 against 16.1.
    constexpr int64_t UNIT = 16384;
    const int64_t units = (N + UNIT - 1) / UNIT;
    int64_t want = std::min({MAX_ITEMS / std::max<int64_t>(T, 1), std::max<int64_t>(10, units / 8), MAX_SEGS, units});
    if (want < 1 || units <= 4) want = 1;
    l.len = (units + want - 1) / want * UNIT;
    l.segs = int((N + l.len - 1) / l.len);
    size_t at = 0;
    auto take = [&](size_t bytes) {
        const size_t p = at;
        at += align256(bytes);
        return p;
    };
    l.rows = std::max<int64_t>(T, 1);
    if (l.segs > 1) {
        l.rows = std::min<int64_t>(l.rows, MAX_ITEMS / l.segs);
        l.keys = take(size_t(l.rows) * l.segs * LIST * 8);
        l.counts = take(size_t(l.rows) * l.segs * 4);
        l.stat = take(size_t(l.rows) * l.segs * 8);
    }
    l.total = std::max<size_t>(at, 256);
    return l;
}

template <bool BF16>
hipError_t launch_rows(const TArgs &a, int64_t rows, hipStream_t st)
{
    const dim3 grid(unsigned(rows * a.segs));
    if (a.segs == 1) {
        hipLaunchKernelGGL((top_rows_kernel<BF16, true>), grid, dim3(TT), 0, st, a);
        return hipGetLastError();
    }
    hipLaunchKernelGGL((top_rows_kernel<BF16, false>), grid, dim3(TT), 0, st, a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(top_join_kernel, dim3(unsigned(rows)), dim3(TT), 0, st, a);
    return hipGetLastError();
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
        e = c.z_dtype == BSQ_BF16 ? launch_rows<true>(a, rows, st) : launch_rows<false>(a, rows, st);
    }
    return e;
}

}  // namespace bsq
