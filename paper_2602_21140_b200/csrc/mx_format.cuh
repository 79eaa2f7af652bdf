// The microscaled 4-bit row format (32 elements share a power-of-two scale).
//
// A row of K elements (K % 32 == 0) is K/2 bytes of codes and K/32 bytes of scales.  Two elements
// share a code byte, the even one in the low half; a code is a sign, two exponent bits and one
// mantissa bit and stands for +-{0, 0.5, 1, 1.5, 2, 3, 4, 6}.  A scale byte s stands for
// 2^(s - 127), 255 for NaN.  Scale rows are padded to a multiple of 16 bytes (mx_scale_pitch) so
// that every row of scales can be read with 16-byte accesses; the padding is never interpreted.
//
// Quantising a block of 32 values x with largest magnitude a:
//   s = clamp(floor(log2 a) - 2 + 127, 0, 254)      (a = 0 gives 0; a NaN or infinity gives 255)
//   code = nearest code of x * 2^(127 - s), ties to the even code, magnitudes above 6 to 6
// so that a * 2^(127 - s) lies in [4, 8): the block uses the whole range of the 4-bit values.  The
// product with a power of two is exact, so the only rounding is the one to 4 bits.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "device_utils.cuh"

namespace moe {

constexpr int kMxBlock = 32;

__host__ __device__ inline int mx_scale_pitch(int cols) { return (cols / kMxBlock + 15) & ~15; }

// Scale byte of a block whose largest magnitude has the fp32 bit pattern `amax_bits` (sign
// clear).  Magnitudes compare like their bit patterns, NaN above infinity.  The exponent field E
// of a normal a is floor(log2 a) + 127; zero and subnormals (E = 0) fall into the clamp.
__device__ __forceinline__ uint32_t mx_scale_byte(uint32_t amax_bits)
{
    const uint32_t e = amax_bits >> 23;
    return e == 255u ? 255u : (e > 2u ? e - 2u : 0u);
}

// 2^(127 - s), normal for every s in [0, 252]; 0 for the NaN scale, which makes the codes of such a
// block (never interpreted as numbers) independent of its contents together with the select below.
__device__ __forceinline__ float mx_inverse_scale(uint32_t s) { return s == 255u ? 0.0f : __uint_as_float((254u - s) << 23); }

// 2^(s - 127): s = 0 is the subnormal 2^-127
__device__ __forceinline__ float mx_scale_value(uint32_t s)
{
    return s == 255u ? __uint_as_float(0x7fc00000u) : __uint_as_float(s ? s << 23 : 0x00400000u);
}

// Eight scaled values to eight codes, element 0 in the lowest four bits.
__device__ __forceinline__ uint32_t mx_pack8(const float (&v)[8])
{
    uint32_t r;
    asm("{\n\t.reg .b8 b0, b1, b2, b3;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 b0, %2, %1;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 b1, %4, %3;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 b2, %6, %5;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 b3, %8, %7;\n\t"
        "mov.b32 %0, {b0, b1, b2, b3};\n\t}"
        : "=r"(r)
        : "f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]), "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7]));
    return r;
}

// Eight codes to their values (exact in fp32).
__device__ __forceinline__ void mx_unpack8(uint32_t c, float (&v)[8])
{
    uint32_t h[4];
    asm("{\n\t.reg .b8 b0, b1, b2, b3;\n\t"
        "mov.b32 {b0, b1, b2, b3}, %4;\n\t"
        "cvt.rn.f16x2.e2m1x2 %0, b0;\n\t"
        "cvt.rn.f16x2.e2m1x2 %1, b1;\n\t"
        "cvt.rn.f16x2.e2m1x2 %2, b2;\n\t"
        "cvt.rn.f16x2.e2m1x2 %3, b3;\n\t}"
        : "=r"(h[0]), "=r"(h[1]), "=r"(h[2]), "=r"(h[3])
        : "r"(c));
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        const float2 f = __half22float2(*reinterpret_cast<const __half2 *>(&h[q]));
        v[2 * q] = f.x; v[2 * q + 1] = f.y;
    }
}

__device__ __forceinline__ uint32_t max_u16x2(uint32_t a, uint32_t b)
{
    uint32_t r;
    asm("max.u16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}

// Largest magnitude of the block as the bit pattern of its 16-bit type: eight elements of this lane, two to a
// word, over the four lanes of an aligned quad.  Magnitudes of 16-bit floats compare like their bit patterns too,
// so this is two instructions per word.
__device__ __forceinline__ uint32_t mx_amax16(const uint4 &u)
{
    uint32_t m = max_u16x2(max_u16x2(u.x & 0x7fff7fffu, u.y & 0x7fff7fffu), max_u16x2(u.z & 0x7fff7fffu, u.w & 0x7fff7fffu));
    m = max_u16x2(m, __shfl_xor_sync(0xffffffffu, m, 1));
    m = max_u16x2(m, __shfl_xor_sync(0xffffffffu, m, 2));
    return max(m & 0xffffu, m >> 16);
}

// Quantise eight consecutive elements held by this lane; the four lanes of an aligned quad hold one
// block.  Every lane of the warp must call it.

// bf16: a bf16 number times a power of two is a bf16 number (down to its subnormals, which are far below half the
// smallest code), so the scaling is done two at a time before they are taken apart.
__device__ __forceinline__ uint32_t mx_quantize8_bf16(const uint4 &u, uint32_t &scale)
{
    scale = mx_scale_byte(mx_amax16(u) << 16);
    const uint32_t inv_bits = __float_as_uint(mx_inverse_scale(scale)) >> 16;
    const uint32_t inv2_bits = inv_bits | (inv_bits << 16);
    const __nv_bfloat162 inv2 = *reinterpret_cast<const __nv_bfloat162 *>(&inv2_bits);
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
    float v[8];
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        const __nv_bfloat162 h = __hmul2(*reinterpret_cast<const __nv_bfloat162 *>(&w[q]), inv2);
        const uint32_t b = *reinterpret_cast<const uint32_t *>(&h);
        v[2 * q] = __uint_as_float(b << 16);
        v[2 * q + 1] = __uint_as_float(b & 0xffff0000u);
    }
    const uint32_t c = mx_pack8(v);
    return scale == 255u ? 0u : c;
}

// fp16: scaled in fp32, whose range the scale may need.
__device__ __forceinline__ uint32_t mx_quantize8_f16(const uint4 &u, uint32_t &scale)
{
    scale = mx_scale_byte(__float_as_uint(__half2float(__ushort_as_half((unsigned short)mx_amax16(u)))) & 0x7fffffffu);
    const float inv = mx_inverse_scale(scale);
    const __half2 *h = reinterpret_cast<const __half2 *>(&u);
    float v[8];
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        const float2 f = __half22float2(h[q]);
        v[2 * q] = f.x * inv; v[2 * q + 1] = f.y * inv;
    }
    const uint32_t c = mx_pack8(v);
    return scale == 255u ? 0u : c;
}

__device__ __forceinline__ uint32_t mx_quantize8_f32(float (&v)[8], uint32_t &scale)
{
    uint32_t a = 0;
#pragma unroll
    for (int q = 0; q < 8; ++q) a = max(a, __float_as_uint(v[q]) & 0x7fffffffu);
    a = max(a, __shfl_xor_sync(0xffffffffu, a, 1));
    a = max(a, __shfl_xor_sync(0xffffffffu, a, 2));
    scale = mx_scale_byte(a);
    const float inv = mx_inverse_scale(scale);
#pragma unroll
    for (int q = 0; q < 8; ++q) v[q] *= inv;
    const uint32_t c = mx_pack8(v);
    return scale == 255u ? 0u : c;
}

// 4 x 4 transpose in a quad of lanes.  Before: w[i] and s[i] belong to this lane's quarter of block 8 i + (lane / 4)
// of the warp's 32 blocks.  After: w holds the whole 16 bytes of block mx_block_of_lane(lane), the result is its scale.
__device__ __forceinline__ int mx_block_of_lane(int lane) { return 8 * (lane & 3) + (lane >> 2); }

__device__ __forceinline__ uint32_t mx_transpose(uint32_t (&w)[4], const uint32_t (&s)[4], int lane)
{
    const unsigned full = 0xffffffffu;
    uint32_t x0 = (lane & 1) ? w[0] : w[1], x1 = (lane & 1) ? w[2] : w[3];
    x0 = __shfl_xor_sync(full, x0, 1); x1 = __shfl_xor_sync(full, x1, 1);
    if (lane & 1) { w[0] = x0; w[2] = x1; } else { w[1] = x0; w[3] = x1; }
    x0 = (lane & 2) ? w[0] : w[2]; x1 = (lane & 2) ? w[1] : w[3];
    x0 = __shfl_xor_sync(full, x0, 2); x1 = __shfl_xor_sync(full, x1, 2);
    if (lane & 2) { w[0] = x0; w[1] = x1; } else { w[2] = x0; w[3] = x1; }
    const int sub = lane & 3;
    return sub == 0 ? s[0] : sub == 1 ? s[1] : sub == 2 ? s[2] : s[3];
}

}  // namespace moe
