// Global norm of many gradient tensors, and their clipping:
//   norm = sqrt(sum over all tensors of g^2),
//   coef = min(1, max_norm / (norm + 1e-6)),  out = coef g.
//
// A prepared table holds the tensors and, for every chunk of CLIP_CHUNK
// elements of a tensor, which tensor it is of, so that one launch walks all
// tensors, small and large, with blocks of equal work.
//
// Both passes are bound by memory (1.0e9 elements, mostly bf16: norm 440 us, 5.6
// TB/s; scaling 935 us, 5.3 TB/s of reads and writes). The squares are summed in fp64 (a sum of
// 1e9 fp32 squares neither overflows nor loses its small terms; at two fp64
// instructions per element the vector units are far from their rate), per
// thread in order of the chunks, then by a fixed tree: no atomics, so a norm
// is the same from run to run.
#include <algorithm>

#include "bsq_internal.h"

namespace bsq {
namespace {

constexpr int CT = 256;                    // threads of a block
constexpr int64_t CLIP_CHUNK = 16384;      // elements
constexpr int64_t CLIP_BLOCKS = 2048;      // partial sums at most

struct ClipEntry {
    const void *src;
    void *dst;
    int64_t n;
    int64_t first;  // its first chunk
    int32_t bf16, vec;
    int64_t pad;
};

// Table buffer: entries [count] | tensor of each chunk [chunks] | partial sums [CLIP_BLOCKS]
struct ClipLayout {
    size_t ent_off, map_off, part_off, total;
};

ClipLayout clip_layout(int64_t count, int64_t chunks)
{
    ClipLayout l{};
    l.ent_off = 0;
    l.map_off = l.ent_off + align256(size_t(count) * sizeof(ClipEntry));
    l.part_off = l.map_off + align256(size_t(chunks) * 4);
    l.total = l.part_off + align256(size_t(CLIP_BLOCKS) * 8);
    return l;
}

// The table is written by kernels from their arguments (no copy from host
// memory, which a captured graph could not hold).
constexpr int ENT_BATCH = 48;
struct EntBatch {
    ClipEntry e[ENT_BATCH];
};

__global__ __launch_bounds__(CT) void clip_table_kernel(ClipEntry *ent, int32_t *map, int64_t at, int count, const EntBatch b)
{
    // one block per tensor: its entry and its chunks' map
    const int i = blockIdx.x;
    if (i >= count) return;
    const ClipEntry e = b.e[i];
    if (threadIdx.x == 0) ent[at + i] = e;
    const int64_t nc = (e.n + CLIP_CHUNK - 1) / CLIP_CHUNK;
    for (int64_t c = threadIdx.x; c < nc; c += CT) map[e.first + c] = int32_t(at + i);
}

struct ClipArgs {
    const ClipEntry *ent;
    const int32_t *map;
    double *part;
    int64_t chunks;
    int nblocks;
    float max_norm;
    float *stats;   // norm, coef
    int32_t *err;
};

__device__ __forceinline__ double block_sum(double v, double *s)
{
    const int t = threadIdx.x, lane = t & 63;
    for (int d = 32; d > 0; d >>= 1) v += __shfl_xor(v, d);
    if (lane == 0) s[t >> 6] = v;
    __syncthreads();
    v = 0.0;
    for (int w = 0; w < CT / 64; ++w) v += s[w];
    return v;
}

__device__ __forceinline__ double square(float f, double acc) { return __builtin_fma(double(f), double(f), acc); }

__global__ __launch_bounds__(CT) void clip_norm_kernel(const ClipArgs a)
{
    __shared__ double s_sum[CT / 64];
    const int t = threadIdx.x;
    double acc = 0.0;
    for (int64_t c = blockIdx.x; c < a.chunks; c += gridDim.x) {
        const ClipEntry e = a.ent[a.map[c]];
        const int64_t i0 = (c - e.first) * CLIP_CHUNK;
        const int n = int(e.n - i0 < CLIP_CHUNK ? e.n - i0 : CLIP_CHUNK);
        if (e.bf16) {
            const uint16_t *p = static_cast<const uint16_t *>(e.src) + i0;
            const int nv = e.vec ? n / 8 : 0;
#pragma unroll 4
            for (int k = t; k < nv; k += CT) {
                const uint4 v = reinterpret_cast<const uint4 *>(p)[k];
                const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    acc = square(__uint_as_float(w[q] << 16), acc);
                    acc = square(__uint_as_float(w[q] & 0xffff0000u), acc);
                }
            }
#pragma unroll 4
            for (int k = 8 * nv + t; k < n; k += CT) acc = square(bf16_to_f32(p[k]), acc);
        } else {
            const float *p = static_cast<const float *>(e.src) + i0;
            const int nv = e.vec ? n / 4 : 0;
#pragma unroll 4
            for (int k = t; k < nv; k += CT) {
                const float4 v = reinterpret_cast<const float4 *>(p)[k];
                acc = square(v.w, square(v.z, square(v.y, square(v.x, acc))));
            }
#pragma unroll 4
            for (int k = 4 * nv + t; k < n; k += CT) acc = square(p[k], acc);
        }
    }
    acc = block_sum(acc, s_sum);
    if (t == 0) a.part[blockIdx.x] = acc;
}

// The norm from the partial sums, in the same order in every block.
__device__ __forceinline__ double clip_total(const ClipArgs &a, double *s)
{
    double v = 0.0;
    for (int k = threadIdx.x; k < a.nblocks; k += CT) v += a.part[k];
    return __builtin_sqrt(block_sum(v, s));
}

// norm and coef; a norm that is not finite clips nothing and is reported. Both
// are judged in fp64: a norm past the range of fp32 is finite, and clips.
__device__ __forceinline__ float clip_stats(const ClipArgs &a, double norm, bool write)
{
    const bool fine = norm - norm == 0.0;
    const double q = double(a.max_norm) / (norm + 1e-6);
    const float coef = (fine && q < 1.0) ? float(q) : 1.0f;
    if (write && threadIdx.x == 0) {
        a.stats[0] = float(norm);
        a.stats[1] = coef;
        if (!fine && a.err) atomicOr(a.err, BSQ_DEVERR_NONFINITE);
    }
    return coef;
}

__global__ __launch_bounds__(CT) void clip_stats_kernel(const ClipArgs a)
{
    __shared__ double s_sum[CT / 64];
    clip_stats(a, clip_total(a, s_sum), true);
}

// out = coef g. Chunks are taken from the last to the first: what the norm
// read last is still in the last-level cache.
__global__ __launch_bounds__(CT) void clip_scale_kernel(const ClipArgs a)
{
    __shared__ double s_sum[CT / 64];
    const int t = threadIdx.x;
    const float coef = clip_stats(a, clip_total(a, s_sum), blockIdx.x == 0);
    for (int64_t r = blockIdx.x; r < a.chunks; r += gridDim.x) {
        const int64_t c = a.chunks - 1 - r;
        const ClipEntry e = a.ent[a.map[c]];
        if (coef == 1.0f && e.src == e.dst) continue;
        const int64_t i0 = (c - e.first) * CLIP_CHUNK;
        const int n = int(e.n - i0 < CLIP_CHUNK ? e.n - i0 : CLIP_CHUNK);
        if (e.bf16) {
            const uint16_t *p = static_cast<const uint16_t *>(e.src) + i0;
            uint16_t *o = static_cast<uint16_t *>(e.dst) + i0;
            const int nv = e.vec ? n / 8 : 0;
#pragma unroll 4
            for (int k = t; k < nv; k += CT) {
                uint4 v = reinterpret_cast<const uint4 *>(p)[k];
                uint32_t w[4] = {v.x, v.y, v.z, v.w};
                if (coef != 1.0f)
#pragma unroll
                    for (int q = 0; q < 4; ++q)
                        w[q] = pack_bf16x2(coef * __uint_as_float(w[q] << 16), coef * __uint_as_float(w[q] & 0xffff0000u));
                reinterpret_cast<uint4 *>(o)[k] = make_uint4(w[0], w[1], w[2], w[3]);
            }
            for (int k = 8 * nv + t; k < n; k += CT) o[k] = (coef == 1.0f) ? p[k] : f32_to_bf16(coef * bf16_to_f32(p[k]));
        } else {
            const float *p = static_cast<const float *>(e.src) + i0;
            float *o = static_cast<float *>(e.dst) + i0;
            const int nv = e.vec ? n / 4 : 0;
#pragma unroll 4
            for (int k = t; k < nv; k += CT) {
                const float4 v = reinterpret_cast<const float4 *>(p)[k];
                reinterpret_cast<float4 *>(o)[k] = make_float4(coef * v.x, coef * v.y, coef * v.z, coef * v.w);
            }
            for (int k = 4 * nv + t; k < n; k += CT) o[k] = coef * p[k];
        }
    }
}

}  // namespace

int64_t clip_chunks(int64_t n) { return (n + CLIP_CHUNK - 1) / CLIP_CHUNK; }

size_t clip_table_bytes(int64_t count, int64_t chunks) { return clip_layout(count, chunks).total; }

hipError_t launch_clip_prepare(int64_t count, const void *const *src, void *const *dst, const int64_t *sizes,
                               const int32_t *dtypes, int64_t chunks, void *table, hipStream_t st)
{
    const ClipLayout l = clip_layout(count, chunks);
    char *tb = static_cast<char *>(table);
    ClipEntry *ent = reinterpret_cast<ClipEntry *>(tb + l.ent_off);
    int32_t *map = reinterpret_cast<int32_t *>(tb + l.map_off);
    int64_t first = 0;
    for (int64_t at = 0; at < count; at += ENT_BATCH) {
        const int nb = int(std::min<int64_t>(ENT_BATCH, count - at));
        EntBatch b{};
        for (int i = 0; i < nb; ++i) {
            ClipEntry &e = b.e[i];
            e.src = src[at + i];
            e.dst = dst ? dst[at + i] : const_cast<void *>(src[at + i]);
            e.n = sizes[at + i];
            e.first = first;
            e.bf16 = dtypes[at + i] == BSQ_BF16;
            e.vec = ((reinterpret_cast<uintptr_t>(e.src) | reinterpret_cast<uintptr_t>(e.dst)) & 15) == 0;
            first += clip_chunks(e.n);
        }
        hipLaunchKernelGGL(clip_table_kernel, dim3(unsigned(nb)), dim3(CT), 0, st, ent, map, at, nb, b);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

hipError_t launch_clip(const bsq_clip_plan &p, bool scale, float max_norm, float *stats, int32_t *err, hipStream_t st)
{
    const ClipLayout l = clip_layout(p.count, p.chunks);
    char *tb = static_cast<char *>(p.table);
    ClipArgs a{};
    a.ent = reinterpret_cast<const ClipEntry *>(tb + l.ent_off);
    a.map = reinterpret_cast<const int32_t *>(tb + l.map_off);
    a.part = reinterpret_cast<double *>(tb + l.part_off);
    a.chunks = p.chunks;
    a.nblocks = int(std::min<int64_t>(std::max<int64_t>(p.chunks, 1), CLIP_BLOCKS));
    a.max_norm = max_norm;
    a.stats = stats;
    a.err = err;
    hipLaunchKernelGGL(clip_norm_kernel, dim3(unsigned(a.nblocks)), dim3(CT), 0, st, a);
    if (scale) hipLaunchKernelGGL(clip_scale_kernel, dim3(unsigned(a.nblocks)), dim3(CT), 0, st, a);
    else hipLaunchKernelGGL(clip_stats_kernel, dim3(1), dim3(CT), 0, st, a);
    return hipGetLastError();
}

}  // namespace bsq
