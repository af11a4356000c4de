// fp32 -> e4m3 codes shared by the kernels that quantise weights (blocks) and activations (rows).
#pragma once
#include <cstdint>

namespace dr {

// two fp32 -> two e4m3 bytes: round to nearest even, saturate to +-448; a NaN of either sign comes out
// as 0x7F (checked against the oracle on sources made of every bit pattern)
__device__ __forceinline__ uint32_t cvt_e4m3x2(float lo, float hi)
{
    uint16_t d;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(d) : "f"(hi), "f"(lo));
    return d;
}
// Eight values of one block row -> eight e4m3 codes of x / scale, packed into two words.
// The codes are first taken from the products with the reciprocal.  Product and true quotient differ by at most
// 2 ulp, so they can round to different codes only (A) next to a midpoint between two codes: the 20 mantissa bits
// e4m3 drops lie within 4 of 0x80000, tested with one multiply-add per value (shifting the 20 bits to the top and
// subtracting (0x80000 - 4) << 12 leaves a value <= 8 << 12) and a min tree; or (B) below 2^-6, where the e4m3
// grid is no longer 3 mantissa bits wide: tested on the packed codes, four at a time (a code of magnitude
// <= small_code = 8 means the product rounded to 2^-6 or less).  In either case all eight are redone with the
// correctly rounded division.  small_code = 0x7F sends every group there (blocks whose reciprocal is not normal).
__device__ __forceinline__ uint2 pack8(const float* t)
{
    const uint32_t h0 = cvt_e4m3x2(t[0], t[1]), h1 = cvt_e4m3x2(t[2], t[3]);
    const uint32_t h2 = cvt_e4m3x2(t[4], t[5]), h3 = cvt_e4m3x2(t[6], t[7]);
    return make_uint2(h0 | (h1 << 16), h2 | (h3 << 16));
}
__device__ __forceinline__ uint2 quantise8(const float* x, float scale, float recip, uint32_t small_code)
{
    float t[8];
    uint32_t d[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        t[k] = __fmul_rn(x[k], recip);
        d[k] = __float_as_uint(t[k]) * 4096u - 0x7FFFC000u;
    }
#pragma unroll
    for (int w = 4; w >= 1; w /= 2)  // min tree (three-input minima were measured and are slower)
#pragma unroll
        for (int k = 0; k < w; ++k) d[k] = min(d[k], d[k + w]);
    const uint32_t dmin = d[0];
    uint2 q = pack8(t);
    // per byte: magnitude + (0x7F - small_code) reaches bit 7 exactly when the magnitude exceeds small_code
    const uint32_t bias = (0x7Fu - small_code) * 0x01010101u;
    const uint32_t big = ((q.x & 0x7F7F7F7Fu) + bias) & ((q.y & 0x7F7F7F7Fu) + bias) & 0x80808080u;
    if (dmin <= 0x8000u || big != 0x80808080u) {
#pragma unroll
        for (int k = 0; k < 8; ++k) t[k] = __fdiv_rn(x[k], scale);
        q = pack8(t);
    }
    return q;
}

// The same codes without a test and a branch: every quotient is corrected.  For kernels that the conversions' and comparisons'
// pipe bounds (the rows of activations: 8192 x 12288 bf16 75 us with the test, 56 without): the tests' integer minima cost more
// there than multiply-adds, and more values are in doubt than in a weight (3.5e-5 of a block's maximum and less is below 2^-6).
//
// x / scale rounded to nearest, from t = x * fl32(1 / scale) by two of Markstein's corrections: the remainder x - t scale is exact in a
// fused multiply-add, and adding it back rounds once; the first makes t faithful, the second correctly rounded.  For
// scales in [2^-100, 2^126], where neither the remainders that can matter (|t| >= 2^-11) nor the reciprocal leave the normal range.
// The caller gives -x, so that the remainder x - t scale comes out negated without another instruction and a zero keeps its
// sign.  PACKED takes two values an instruction: 3 % less time from bf16, where instructions bound (8192 x 12288: 54.8 against
// 56.1 us), 12 % more from fp32, where the memory does (81.6 against 72.8).
__device__ __forceinline__ uint64_t two_of(float lo, float hi)
{
    uint64_t d;
    asm("mov.b64 %0, {%1, %2};" : "=l"(d) : "f"(lo), "f"(hi));
    return d;
}
__device__ __forceinline__ uint64_t fma_two(uint64_t a, uint64_t b, uint64_t c)
{
    uint64_t d;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
    return d;
}
__device__ __forceinline__ uint64_t mul_two(uint64_t a, uint64_t b)
{
    uint64_t d;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
    return d;
}
__device__ __forceinline__ uint64_t add_two(uint64_t a, uint64_t b)
{
    uint64_t d;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
    return d;
}
template <bool PACKED>
__device__ __forceinline__ uint2 quantise8_corrected(const float* minus_x, float scale, float recip)
{
    float t[8];
    const bool in_range = scale >= 7.8886091e-31f && scale <= 8.5070592e+37f;
    if (!PACKED && in_range) {
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            t[k] = __fmul_rn(minus_x[k], -recip);
            t[k] = fmaf(fmaf(t[k], scale, minus_x[k]), -recip, t[k]);
            t[k] = fmaf(fmaf(t[k], scale, minus_x[k]), -recip, t[k]);
        }
    } else if (in_range) {
        const uint64_t minus_r = two_of(-recip, -recip), s = two_of(scale, scale);
#pragma unroll
        for (int k = 0; k < 8; k += 2) {
            const uint64_t nx = two_of(minus_x[k], minus_x[k + 1]);
            uint64_t q = mul_two(nx, minus_r);
            q = fma_two(fma_two(q, s, nx), minus_r, q);
            q = fma_two(fma_two(q, s, nx), minus_r, q);
            asm("mov.b64 {%0, %1}, %2;" : "=f"(t[k]), "=f"(t[k + 1]) : "l"(q));
        }
    } else {
#pragma unroll
        for (int k = 0; k < 8; ++k) t[k] = __fdiv_rn(-minus_x[k], scale);
    }
    return pack8(t);
}

// Stored scale of a block whose largest magnitude is m: m / 448 held inside the normal fp32 range, so that a block whose
// m / 448 underflows (the all-zero block among them) and a block holding an infinity keep finite, normal scales.
__device__ __forceinline__ float scale_of(float m)
{
    return fminf(fmaxf(__fdiv_rn(m, 448.0f), 1.17549435e-38f), 3.40282347e+38f);
}
// quantise8's last argument for a block of this reciprocal scale.
__device__ __forceinline__ uint32_t small_code_of(float recip) { return recip >= 1.17549435e-38f ? 8u : 0x7Fu; }

}  // namespace dr
