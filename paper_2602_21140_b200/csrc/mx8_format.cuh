// The microscaled 8-bit row format in which activations are kept for a backward pass (32 elements share a power-of-two scale).
//
// A row of K elements (K % 32 == 0) is K bytes of codes, e4m3 floats (a sign, four exponent bits, three of mantissa, largest
// 448), and scale bytes as in mx_format.cuh: s stands for 2^(s - 127), 255 for NaN, rows of scales mx_scale_pitch apart.
//
// Quantising a block of 32 values x with largest magnitude a:
//   s = the smallest of 0 .. 254 with a <= 448 * 2^(s - 127)     (a NaN or infinity gives 255 and codes 0)
//   code = nearest code of x * 2^(127 - s), ties to even
// so nothing saturates, and a block uses the top binade of the codes: x is off by at most 2^-4 of itself, or 2^-10 of the scale where
// that is more (below 2^-6 of the scale the codes are multiples of 2^-9 of it, so what is below 2^-10 of it becomes 0).  (The 4-bit format lets the block's largest values saturate instead; here that would cost up to an eighth of a
// gradient's largest terms.)  The product with a power of two is exact, so the only rounding is the one to 8 bits.
#pragma once

#include "mx_format.cuh"

namespace moe {

// Scale byte of a block whose largest magnitude has the fp32 bit pattern `amax_bits` (sign clear).  448 = 1.75 * 2^8: a
// mantissa above 1.75 needs the next power of two.
__device__ __forceinline__ uint32_t mx8_scale_byte(uint32_t amax_bits)
{
    const uint32_t e = (amax_bits + 0x1fffffu) >> 23;          // exponent field, one more if the mantissa is above 1.75
    return amax_bits >= 0x7f800000u ? 255u : (e > 8u ? e - 8u : 0u);
}

// Four scaled values (within 448) to four codes, element 0 in the lowest byte.
__device__ __forceinline__ uint32_t mx8_pack4(float a, float b, float c, float d)
{
    uint32_t r;
    asm("{\n\t.reg .b16 lo, hi;\n\t"
        "cvt.rn.satfinite.e4m3x2.f32 lo, %2, %1;\n\t"
        "cvt.rn.satfinite.e4m3x2.f32 hi, %4, %3;\n\t"
        "mov.b32 %0, {lo, hi};\n\t}"
        : "=r"(r)
        : "f"(a), "f"(b), "f"(c), "f"(d));
    return r;
}

// Four codes to their values (exact in fp16 and so in fp32).
__device__ __forceinline__ void mx8_unpack4(uint32_t c, float *v)
{
    uint32_t h[2];
    asm("{\n\t.reg .b16 lo, hi;\n\t"
        "mov.b32 {lo, hi}, %2;\n\t"
        "cvt.rn.f16x2.e4m3x2 %0, lo;\n\t"
        "cvt.rn.f16x2.e4m3x2 %1, hi;\n\t}"
        : "=r"(h[0]), "=r"(h[1])
        : "r"(c));
#pragma unroll
    for (int q = 0; q < 2; ++q) {
        const float2 f = __half22float2(*reinterpret_cast<const __half2 *>(&h[q]));
        v[2 * q] = f.x; v[2 * q + 1] = f.y;
    }
}

// Largest magnitude of eight values as a bit pattern (NaN above infinity).
__device__ __forceinline__ uint32_t mx8_amax(const float (&v)[8])
{
    uint32_t a = 0;
#pragma unroll
    for (int q = 0; q < 8; ++q) a = max(a, __float_as_uint(v[q]) & 0x7fffffffu);
    return a;
}

// Eight values of a block with scale byte s.
__device__ __forceinline__ uint2 mx8_quantize8(const float (&v)[8], uint32_t s)
{
    const float inv = mx_inverse_scale(s);
    const uint2 c = make_uint2(mx8_pack4(v[0] * inv, v[1] * inv, v[2] * inv, v[3] * inv),
                               mx8_pack4(v[4] * inv, v[5] * inv, v[6] * inv, v[7] * inv));
    return s == 255u ? make_uint2(0u, 0u) : c;
}

}  // namespace moe
