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

// 2^-e for a finite block's scale byte (0 .. 253): exponent field 254 - byte, never subnormal.
__device__ __forceinline__ float mx_inverse(uint32_t byte) { return __uint_as_float((254u - byte) << 23); }

// 2^e.
__device__ __forceinline__ float mx_scale_value(uint32_t byte)
{
    return byte == 255u ? __uint_as_float(0x7FFFFFFFu) : byte == 0u ? __uint_as_float(0x00400000u) : __uint_as_float(byte << 23);
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

// c + a * b of two values at once.
__device__ __forceinline__ void fma_pair(float a0, float a1, float b, float c, float &r0, float &r1)
{
    uint64_t x, y, z, r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(x) : "f"(a0), "f"(a1));
    asm("mov.b64 %0, {%1, %1};" : "=l"(y) : "f"(b));
    asm("mov.b64 %0, {%1, %1};" : "=l"(z) : "f"(c));
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(x), "l"(y), "l"(z));
    asm("mov.b64 {%0, %1}, %2;" : "=f"(r0), "=f"(r1) : "l"(r));
}

// Byte B of each of four words, in their order.
template <int B> __device__ __forceinline__ uint32_t same_byte(uint32_t w0, uint32_t w1, uint32_t w2, uint32_t w3)
{
    constexpr uint32_t sel = B | (4 + B) << 4;
    return __byte_perm(__byte_perm(w0, w1, sel), __byte_perm(w2, w3, sel), 0x5410);
}

// Magnitude codes (bits 0 to 2 of `code`; what lies above is a constant) of two values of magnitude a * inv in [0, 6], rounded up
// iff h < rint(p * 2^16); `draws` holds the two h.  The codes' values 0, 0.5 .. 2, 3, 4, 6 are the places where a concave function
// of three pieces takes whole numbers: with a' = a * inv it is half of min(2 a', a' + 2, a' / 2 + 4) (slopes 2, 1, 1/2 up to 2, 4,
// 6).  Each piece plus 64 is one fused multiply-add with a single rounding, to 2^-17, ties to even: the minimum is
// 64 + (code + rint(p * 2^16) / 2^16) / 2.  A draw put into the mantissa of 64 is 64 + h / 2^17; the difference is exact, and
// rounding it up to a multiple of one half (the last place of 2^22 + 64, which a difference down to -1/2 does not leave) rounds
// the code up iff h is below the fraction.  (Integer additions and shifts in place of the last two steps take 1 to 2 % longer: the
// integer pipe, which gathers and masks, is the busier one.  Single instead of paired multiply-adds: 3 % longer.)
__device__ __forceinline__ void e2m1_stochastic_pair(float a0, float a1, float inv, uint32_t draws, uint32_t &code0, uint32_t &code1)
{
    float s0, s1, t0, t1, u0, u1;
    fma_pair(a0, a1, inv, 64.0f, s0, s1);
    fma_pair(a0, a1, 0.5f * inv, 65.0f, t0, t1);
    fma_pair(a0, a1, 0.25f * inv, 66.0f, u0, u1);
    asm("min.f32 %0, %0, %1, %2;" : "+f"(s0) : "f"(t0), "f"(u0));
    asm("min.f32 %0, %0, %1, %2;" : "+f"(s1) : "f"(t1), "f"(u1));
    const uint32_t h0 = __byte_perm(draws, 0x42800000u, 0x7610), h1 = __byte_perm(draws, 0x42800000u, 0x7632);
    uint64_t x, y, r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(x) : "f"(s0), "f"(s1));
    asm("mov.b64 %0, {%1, %2};" : "=l"(y) : "r"(h0), "r"(h1));
    asm("sub.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(x), "l"(y));
    asm("mov.b64 %0, {%1, %1};" : "=l"(y) : "f"(4194368.0f));
    asm("add.rp.f32x2 %0, %1, %2;" : "=l"(r) : "l"(r), "l"(y));
    asm("mov.b64 {%0, %1}, %2;" : "=r"(code0), "=r"(code1) : "l"(r));
}

// Eight neighbouring values as they lie in memory.
template <int DT> struct Eight;
template <> struct Eight<UQ_BF16> {
    uint32_t w[4];
    __device__ __forceinline__ uint32_t max_abs_bits() const              // of the binary32 values
    {
        uint32_t m = w[0] & 0x7FFF7FFFu;
#pragma unroll
        for (int t = 1; t < 4; ++t) m = __vmaxu2(m, w[t] & 0x7FFF7FFFu);
        return max(m << 16, m & 0xFFFF0000u);
    }
    __device__ __forceinline__ void values(float (&v)[8]) const
    {
#pragma unroll
        for (int t = 0; t < 4; ++t) { v[2 * t] = bf16lo(w[t]); v[2 * t + 1] = bf16hi(w[t]); }
    }
    __device__ __forceinline__ void magnitudes(float (&v)[8]) const
    {
#pragma unroll
        for (int t = 0; t < 4; ++t) { v[2 * t] = bf16lo(w[t] & 0x7FFF7FFFu); v[2 * t + 1] = bf16hi(w[t] & 0x7FFF7FFFu); }
    }
    // signs in bit 7 of the bytes: of elements 0, 2, 4, 6 and of 1, 3, 5, 7
    __device__ __forceinline__ uint32_t even_signs() const { return same_byte<1>(w[0], w[1], w[2], w[3]); }
    __device__ __forceinline__ uint32_t odd_signs() const { return same_byte<3>(w[0], w[1], w[2], w[3]); }
};
template <> struct Eight<UQ_F32> {
    uint32_t w[8];
    __device__ __forceinline__ uint32_t max_abs_bits() const
    {
        uint32_t m = 0;
#pragma unroll
        for (int t = 0; t < 8; ++t) m = max(m, w[t] & 0x7FFFFFFFu);
        return m;
    }
    __device__ __forceinline__ void values(float (&v)[8]) const
    {
#pragma unroll
        for (int t = 0; t < 8; ++t) v[t] = __uint_as_float(w[t]);
    }
    __device__ __forceinline__ void magnitudes(float (&v)[8]) const
    {
#pragma unroll
        for (int t = 0; t < 8; ++t) v[t] = __uint_as_float(w[t] & 0x7FFFFFFFu);
    }
    __device__ __forceinline__ uint32_t even_signs() const { return same_byte<3>(w[0], w[2], w[4], w[6]); }
    __device__ __forceinline__ uint32_t odd_signs() const { return same_byte<3>(w[1], w[3], w[5], w[7]); }
};

// A lane's eight values of a block that it shares with three neighbouring lanes: its codes, and the block's scale byte.  draws:
// word t holds those of elements 2 t and 2 t + 1, low half first.  The warp is converged.
template <int DT, bool SR> __device__ __forceinline__ uint32_t quantize_eight(const Eight<DT> &x, const uint4 &draws, uint32_t &byte)
{
    uint32_t m = x.max_abs_bits();
    m = max(m, __shfl_xor_sync(0xFFFFFFFFu, m, 1));
    m = max(m, __shfl_xor_sync(0xFFFFFFFFu, m, 2));
    byte = mx_scale_byte(m);
    const float inv = mx_inverse(byte);                    // (of a block that is not finite: anything)
    uint32_t codes;
    float v[8];
    if constexpr (SR) {
        const uint32_t h[4] = {draws.x, draws.y, draws.z, draws.w};
        uint32_t c[8];
        x.magnitudes(v);
#pragma unroll
        for (int t = 0; t < 4; ++t) e2m1_stochastic_pair(v[2 * t], v[2 * t + 1], inv, h[t], c[2 * t], c[2 * t + 1]);
        const uint32_t even = same_byte<0>(c[0], c[2], c[4], c[6]), odd = same_byte<0>(c[1], c[3], c[5], c[7]);
        codes = (even & 0x07070707u) | ((x.even_signs() >> 4) & 0x08080808u) | ((odd << 4) & 0x70707070u) | (x.odd_signs() & 0x80808080u);
    } else {
        x.values(v);
#pragma unroll
        for (int t = 0; t < 4; ++t) mul_pair(v[2 * t], v[2 * t + 1], inv, inv, v[2 * t], v[2 * t + 1]);
        codes = e2m1x8_nearest(v);
    }
    return byte == 255u ? 0u : codes;
}

// The value of a 4-bit code: magnitude bits in the top of a binary32 subnormal or small normal, times 2^126 (exact).
__device__ __forceinline__ float mx_code_value(uint32_t code)
{
    return __uint_as_float(((code & 8u) << 28) | ((code & 7u) << 22)) * __uint_as_float(253u << 23);
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
