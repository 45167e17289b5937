// Rows of a vocabulary's logits in bf16 or fp32, read eight words at a time, and
// powers of two in 64 bits: shared by the kernels that reduce such rows
// (top.hip, draft.hip, distill.hip).
#pragma once

#include "bsq_internal.h"

namespace bsq {
namespace {

typedef uint32_t vr_u32x4_t __attribute__((ext_vector_type(4)));
// sixteen bytes at the alignment of their elements (rows of an odd length)
typedef vr_u32x4_t vr_bf16x8_raw_t __attribute__((aligned(2)));
typedef vr_u32x4_t vr_f32x4_raw_t __attribute__((aligned(4)));

// Eight words of a row from `at` on, as they are stored.
template <bool BF16>
struct Words8 {
    vr_u32x4_t raw[BF16 ? 1 : 2];

    // words [at, at + 8) of `row`
    template <typename Int>
    __device__ __forceinline__ void load(const void *row, Int at)
    {
        if constexpr (BF16) {
            raw[0] = *reinterpret_cast<const vr_bf16x8_raw_t *>(static_cast<const uint16_t *>(row) + at);
        } else {
            const vr_f32x4_raw_t *p = reinterpret_cast<const vr_f32x4_raw_t *>(static_cast<const float *>(row) + at);
            raw[0] = p[0];
            raw[1] = p[1];
        }
    }

    // likewise; those from `end` on are -inf
    template <typename Int>
    __device__ __forceinline__ void load(const void *row, Int at, Int end)
    {
        if (at + 8 <= end) {
            load(row, at);
            return;
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const bool in = at + e < end;
            if constexpr (BF16) {
                const uint32_t v = in ? static_cast<const uint16_t *>(row)[at + e] : 0xff80u;
                if (e & 1) raw[0][e >> 1] |= v << 16;
                else raw[0][e >> 1] = v;
            } else {
                raw[e >> 2][e & 3] = in ? static_cast<const uint32_t *>(row)[at + e] : 0xff800000u;
            }
        }
    }

    __device__ __forceinline__ float operator[](int e) const
    {
        if constexpr (BF16) return __uint_as_float((e & 1) ? raw[0][e >> 1] & 0xffff0000u : raw[0][e >> 1] << 16);
        else return __uint_as_float(raw[e >> 2][e & 3]);
    }
};

template <bool BF16>
__device__ __forceinline__ float word_at(const void *row, int64_t i)
{
    if constexpr (BF16) return bf16_to_f32(static_cast<const uint16_t *>(row)[i]);
    else return static_cast<const float *>(row)[i];
}

// 2^(d c) in 64 bits, for products from -2000 to 1000; NaN for a NaN.
// d c = n + f, |f| <= 1/2: n by adding 1.5 2^52, f with one rounding; 2^f = 1 + f g(f), g the
// polynomial of degree 8 through its Chebyshev nodes (3.7e-14 of the value: of a draw from
// 151936 words one in some 10^8 is another word for it; 1 at 0). 13 instructions of 64
// bits, 32 with the constants' moves; the library's exp2 compiles to 19 and 42.
__device__ __forceinline__ double exp2_64(double d, double c)
{
    constexpr double SHIFT = 6755399441055744.0;
    const double t = __builtin_fma(d, c, SHIFT);
    const double f = __builtin_fma(d, c, SHIFT - t);
    double g = 0x1.b63880a30e9ffp-24;
    g = __builtin_fma(g, f, 0x1.63d136366db24p-20);
    g = __builtin_fma(g, f, 0x1.ffcb9515a8016p-17);
    g = __builtin_fma(g, f, 0x1.4308ac85aa947p-13);
    g = __builtin_fma(g, f, 0x1.5d87fe86fe88ep-10);
    g = __builtin_fma(g, f, 0x1.3b2ab7181b755p-7);
    g = __builtin_fma(g, f, 0x1.c6b08d7047e52p-5);
    g = __builtin_fma(g, f, 0x1.ebfbdff823cedp-3);
    g = __builtin_fma(g, f, 0x1.62e42fefa39efp-1);
    g = __builtin_fma(g, f, 1.0);
    return __builtin_ldexp(g, int(uint32_t(__builtin_bit_cast(uint64_t, t))));
}

// 2^((z - ref) c) of logits z up to ref, c > 0. What is more than 1000 / c below ref (-inf
// among it) is 0; NaN for a NaN, and where ref and z are +inf. (-inf as ref counts as 0.)
struct Exp2Below {
    double ref, c;
    float lowest;
    uint32_t far;  // high word of -1500 / c: 2^-1500 is 0
    // reach: 1000 / c
    __device__ __forceinline__ Exp2Below(float m, double scale, double reach) : c(scale)
    {
        const float r = m == -__builtin_inff() ? 0.0f : m;
        ref = double(r);
        const float low = float(ref - reach);
        lowest = low > -__FLT_MAX__ ? low : -__FLT_MAX__;
        far = uint32_t(__builtin_bit_cast(uint64_t, -1.5 * reach) >> 32);
    }
    __device__ __forceinline__ Exp2Below(float m, double scale) : Exp2Below(m, scale, 1000.0 / scale) {}
    __device__ __forceinline__ double operator()(float z) const
    {
        uint64_t d = __builtin_bit_cast(uint64_t, double(z) - ref);
        d = (uint64_t(z < lowest ? far : uint32_t(d >> 32)) << 32) | uint32_t(d);
        return exp2_64(__builtin_bit_cast(double, d), c);
    }
};

// Inclusive scans of a wave by data-parallel moves (rows of 16 lanes, then a row's last
// lane into the next row, lane 31 into the upper half): lane 63 ends with all of it. A few
// cycles a step, where a shuffle through LDS takes some hundred.
template <int CTRL, int ROWS, typename T>
__device__ __forceinline__ T moved(T v, T none)
{
    if constexpr (sizeof(T) == 8) {
        const uint64_t a = __builtin_bit_cast(uint64_t, v), o = __builtin_bit_cast(uint64_t, none);
        const uint32_t lo = __builtin_amdgcn_update_dpp(int(uint32_t(o)), int(uint32_t(a)), CTRL, ROWS, 0xf, false);
        const uint32_t hi = __builtin_amdgcn_update_dpp(int(uint32_t(o >> 32)), int(uint32_t(a >> 32)), CTRL, ROWS, 0xf, false);
        return __builtin_bit_cast(T, (uint64_t(hi) << 32) | lo);
    } else {
        return __builtin_bit_cast(T, __builtin_amdgcn_update_dpp(__builtin_bit_cast(int, none), __builtin_bit_cast(int, v), CTRL,
                                                                 ROWS, 0xf, false));
    }
}

template <typename T, typename Op>
__device__ __forceinline__ T wave_scan(T v, T none, Op op)
{
    v = op(moved<0x111, 0xf>(v, none), v);  // from 1, 2, 4 and 8 lanes below in the row
    v = op(moved<0x112, 0xf>(v, none), v);
    v = op(moved<0x114, 0xf>(v, none), v);
    v = op(moved<0x118, 0xf>(v, none), v);
    v = op(moved<0x142, 0xa>(v, none), v);  // lane 15 of a row into rows 1 and 3
    v = op(moved<0x143, 0xc>(v, none), v);  // lane 31 into rows 2 and 3
    return v;
}

template <typename T>
__device__ __forceinline__ T lane_value(T v, int lane)
{
    if constexpr (sizeof(T) == 8) {
        const uint64_t a = __builtin_bit_cast(uint64_t, v);
        const uint32_t lo = __builtin_amdgcn_readlane(int(uint32_t(a)), lane), hi = __builtin_amdgcn_readlane(int(uint32_t(a >> 32)), lane);
        return __builtin_bit_cast(T, (uint64_t(hi) << 32) | lo);
    } else {
        return __builtin_bit_cast(T, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), lane));
    }
}

template <typename T>
__device__ __forceinline__ T wave_sum(T v)
{
    return lane_value(wave_scan(v, T(0), [](T a, T b) { return a + b; }), 63);
}

// (NaN counts as nothing)
__device__ __forceinline__ float wave_max(float v)
{
    return lane_value(wave_scan(v, -__builtin_inff(), [](float a, float b) { return fmaxf(a, b); }), 63);
}

}  // namespace
}  // namespace bsq
