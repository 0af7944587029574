// Microscaled 4-bit values: the arithmetic that the quantizing kernels share.
//
// A block is 32 values of a row.  With A its largest magnitude, e is the smallest integer >= -127 with A <= 6 * 2^e, and a
// value x becomes the E2M1 number (0, 0.5, 1, 1.5, 2, 3, 4, 6 with a sign) that x / 2^e is rounded to.  Since e covers A, nothing
// saturates, so the stochastic rounding is unbiased.  2^e is a power of two: x / 2^e, the neighbours' distances and the ties are
// exact in binary32, and a code is decided without a rounded intermediate.
#pragma once

#include "uq_device.cuh"

namespace uq {

constexpr uint32_t kMxTag = 0x4D584634u;      // fourth counter word of the draws; the gradient quantizers use 0
constexpr int kMxTile = 128;                  // a scale tile: 128 rows x 4 blocks of 32 columns, 512 bytes

__host__ __device__ __forceinline__ int64_t mx_blocks(int64_t cols) { return (cols + 31) >> 5; }
__host__ __device__ __forceinline__ int64_t mx_ktiles(int64_t cols) { return (cols + kMxTile - 1) / kMxTile; }

// Where the scale of (row, block) lies.
__host__ __device__ __forceinline__ int64_t mx_scale_at(int64_t row, int64_t block, int64_t ktiles)
{
    return ((row >> 7) * ktiles + (block >> 2)) * 512 + (row & 31) * 16 + ((row >> 5) & 3) * 4 + (block & 3);
}

// The scale byte (e + 127) for a block's largest magnitude, given as its binary32 bits; 255 (E8M0's NaN) if not finite.
// A <= 1.5 * 2^(e+2): adding 2^22 - 1 to the bits carries into the exponent iff the mantissa is above 1.5.
__device__ __forceinline__ uint32_t mx_scale_byte(uint32_t amax_bits)
{
    if (amax_bits >= 0x7F800000u) return 255u;
    const uint32_t up = (amax_bits + 0x3FFFFFu) >> 23;
    return up > 2u ? up - 2u : 0u;
}

// 2^-e for a finite block's scale byte (0 .. 252): exponent field 254 - byte, never subnormal.
__device__ __forceinline__ float mx_inverse(uint32_t byte) { return __uint_as_float((254u - byte) << 23); }

// 2^e.
__device__ __forceinline__ float mx_scale_value(uint32_t byte)
{
    return byte == 255u ? __uint_as_float(0x7FFFFFFFu) : byte == 0u ? __uint_as_float(0x00400000u) : __uint_as_float(byte << 23);
}

// The value of a 4-bit code: magnitude bits in the top of a binary32 subnormal or small normal, times 2^126 (exact).
__device__ __forceinline__ float mx_code_value(uint32_t code)
{
    return __uint_as_float(((code & 8u) << 28) | ((code & 7u) << 22)) * __uint_as_float(253u << 23);
}

// Magnitude code of a in [0, 6], rounded up iff h < rint(p * 2^16).  With u = 0.5, 1 or 2 the grid's step at a, adding
// 2^23 * (u / 2^16) leaves rint(a / u * 2^16) in the sum's low bits (one rounding, ties to even); steps before this binade
// are added as 2 * 2^16 per binade, and 2^16 - 1 - h carries into the code iff h is below the fraction.
__device__ __forceinline__ uint32_t e2m1_stochastic(float a, uint32_t h)
{
    const uint32_t e = max(__float_as_uint(a) & 0x7F800000u, 0x3F800000u), magic = e + (6u << 23);
    const uint32_t t = __float_as_uint(__fadd_rn(a, __uint_as_float(magic))) - magic + ((e - 0x3F800000u) >> 6);
    return (t + 65535u - h) >> 16;
}

// Eight values rounded to the nearest code, ties to the even one (the conversion's own rule), element 0 in the low bits.
__device__ __forceinline__ uint32_t e2m1x8_nearest(const float (&v)[8])
{
    uint32_t r;
    asm("{\n\t.reg .b8 b0, b1, b2, b3;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 b0, %2, %1;\n\tcvt.rn.satfinite.e2m1x2.f32 b1, %4, %3;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 b2, %6, %5;\n\tcvt.rn.satfinite.e2m1x2.f32 b3, %8, %7;\n\t"
        "mov.b32 %0, {b0, b1, b2, b3};\n\t}"
        : "=r"(r) : "f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]), "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7]));
    return r;
}

// Eight values with their 16-bit draws (word t holds those of elements 2 t and 2 t + 1, low half first).
__device__ __forceinline__ uint32_t e2m1x8_stochastic(const float (&v)[8], const uint4 &draws)
{
    const uint32_t w[4] = {draws.x, draws.y, draws.z, draws.w};
    uint32_t r = 0;
#pragma unroll
    for (int t = 0; t < 8; ++t) {
        const uint32_t h = (t & 1) ? w[t >> 1] >> 16 : w[t >> 1] & 0xFFFFu;
        const uint32_t code = e2m1_stochastic(fabsf(v[t]), h) | ((__float_as_uint(v[t]) >> 28) & 8u);
        r |= code << (4 * t);
    }
    return r;
}

__device__ __forceinline__ uint32_t abs_bits(float v) { return __float_as_uint(v) & 0x7FFFFFFFu; }

__device__ __forceinline__ uint32_t max_abs_bits(const float (&v)[8])
{
    uint32_t m = 0;
#pragma unroll
    for (int t = 0; t < 8; ++t) m = max(m, abs_bits(v[t]));
    return m;
}

// Eight consecutive values of a row, of which the first `n` exist (the others are 0).  `wide`: the address is 16-byte aligned.
template <int DT> __device__ __forceinline__ void load8(const void *base, int64_t at, int n, bool wide, float (&v)[8])
{
    if (n >= 8 && wide) {
        const uint4 q = ld_stream((const char *)base + at * Elem<DT>::BYTES);
        if constexpr (DT == UQ_BF16) {
            Elem<UQ_BF16>::unpack(q, v);
        } else {
            const uint4 q2 = ld_stream((const char *)base + at * 4 + 16);
            float lo[4], hi[4];
            Elem<UQ_F32>::unpack(q, lo);
            Elem<UQ_F32>::unpack(q2, hi);
#pragma unroll
            for (int t = 0; t < 4; ++t) { v[t] = lo[t]; v[4 + t] = hi[t]; }
        }
        return;
    }
#pragma unroll
    for (int t = 0; t < 8; ++t) {
        v[t] = 0.0f;
        if (t < n) {
            if constexpr (DT == UQ_BF16) v[t] = __uint_as_float((uint32_t)__ldg((const unsigned short *)base + at + t) << 16);
            else v[t] = __ldg((const float *)base + at + t);
        }
    }
}

// binary32 to bf16 bits, to nearest, ties to even; NaN stays NaN.
__device__ __forceinline__ uint32_t bf16_bits(float v)
{
    unsigned short r;
    asm("cvt.rn.bf16.f32 %0, %1;" : "=h"(r) : "f"(v));
    return r;
}
__device__ __forceinline__ uint32_t bf16x2_bits(float lo, float hi)
{
    uint32_t r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}

template <int DT> __device__ __forceinline__ void store1(void *base, int64_t at, float v)
{
    if constexpr (DT == UQ_BF16) ((unsigned short *)base)[at] = (unsigned short)bf16_bits(v);
    else ((float *)base)[at] = v;
}

template <int DT> __device__ __forceinline__ void store8(void *base, int64_t at, int n, bool wide, const float (&v)[8])
{
    if (n >= 8 && wide) {
        if constexpr (DT == UQ_BF16) {
            *(uint4 *)((char *)base + at * 2) = make_uint4(bf16x2_bits(v[0], v[1]), bf16x2_bits(v[2], v[3]), bf16x2_bits(v[4], v[5]),
                                                           bf16x2_bits(v[6], v[7]));
        } else {
            *(float4 *)((float *)base + at) = make_float4(v[0], v[1], v[2], v[3]);
            *(float4 *)((float *)base + at + 4) = make_float4(v[4], v[5], v[6], v[7]);
        }
        return;
    }
#pragma unroll
    for (int t = 0; t < 8; ++t)
        if (t < n) store1<DT>(base, at + t, v[t]);
}

}  // namespace uq
