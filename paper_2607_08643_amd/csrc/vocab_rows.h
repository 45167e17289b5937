// Rows of a vocabulary's logits in bf16 or fp32, read eight words at a time, and
// powers of two in 64 bits: shared by the kernels that reduce such rows
// (top.hip, draft.hip).
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

    // words [at, at + 8) of `row`; those from `end` on are -inf
    __device__ __forceinline__ void load(const void *row, int64_t at, int64_t end)
    {
        if (at + 8 <= end) {
            if constexpr (BF16) {
                raw[0] = *reinterpret_cast<const vr_bf16x8_raw_t *>(static_cast<const uint16_t *>(row) + at);
            } else {
                const vr_f32x4_raw_t *p = reinterpret_cast<const vr_f32x4_raw_t *>(static_cast<const float *>(row) + at);
                raw[0] = p[0];
                raw[1] = p[1];
            }
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

// 2^x in 64 bits for x up to 1000; 0 below -1000 (-inf among it), NaN for NaN.
// x = n + f, |f| <= 1/2, n by adding 1.5 2^52; 2^f by the polynomial of degree 10
// through its Chebyshev nodes (3.2e-16 of the value), n added to the exponent. Ten fma
// beside some six other instructions: a library exp takes about three times as many.
__device__ __forceinline__ double exp2_64(double x)
{
    constexpr double SHIFT = 6755399441055744.0;
    const double t = x + SHIFT;
    const double f = x - (t - SHIFT);
    double p = 0x1.e6063f7217bc6p-28;
    p = __builtin_fma(p, f, 0x1.b675bca4eeebbp-24);
    p = __builtin_fma(p, f, 0x1.62bfd47773353p-20);
    p = __builtin_fma(p, f, 0x1.ffcb54062e698p-17);
    p = __builtin_fma(p, f, 0x1.430913096fd9fp-13);
    p = __builtin_fma(p, f, 0x1.5d87fe9d7a584p-10);
    p = __builtin_fma(p, f, 0x1.3b2ab6fba1ddap-7);
    p = __builtin_fma(p, f, 0x1.c6b08d703ce49p-5);
    p = __builtin_fma(p, f, 0x1.ebfbdff82c598p-3);
    p = __builtin_fma(p, f, 0x1.62e42fefa3a19p-1);
    p = __builtin_fma(p, f, 1.0);
    const uint64_t b = __builtin_bit_cast(uint64_t, p);
    const uint32_t hi = uint32_t(b >> 32) + (uint32_t(__builtin_bit_cast(uint64_t, t)) << 20);
    const double r = __builtin_bit_cast(double, (uint64_t(hi) << 32) | uint32_t(b));
    return x < -1000.0 ? 0.0 : r;
}

}  // namespace
}  // namespace bsq
