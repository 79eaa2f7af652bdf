// moe_mx_quantize / moe_mx_dequantize: rows to the microscaled 4-bit format and back; moe_kept_dequantize: back from 8 bits.
//
// Both are one pass over the data and bound by HBM: n elements of `size` bytes are read (written)
// once and n * 17/32 bytes written (read).  A thread owns eight consecutive elements (one 16-byte
// access of a 16-bit type) and four neighbouring lanes own a block, so the block's largest
// magnitude takes two shuffles.  Units of eight
// elements are numbered through all rows, so short rows fill the warps as well as long ones.
#include "../../include/moe_route.h"

#include "mx8_format.cuh"

namespace {

using namespace moe;

constexpr int kRowThreads = 256;

template <int DT> struct Elem;
template <> struct Elem<MOE_DTYPE_BF16> { static constexpr int kVec = 1; };
template <> struct Elem<MOE_DTYPE_F16> { static constexpr int kVec = 1; };
template <> struct Elem<MOE_DTYPE_F32> { static constexpr int kVec = 2; };

template <int DT>
__device__ __forceinline__ uint32_t quantize8(const uint4 (&u)[Elem<DT>::kVec], uint32_t &scale)
{
    if constexpr (DT == MOE_DTYPE_BF16) {
        return mx_quantize8_bf16(u[0], scale);
    } else if constexpr (DT == MOE_DTYPE_F16) {
        return mx_quantize8_f16(u[0], scale);
    } else {
        const float *f = reinterpret_cast<const float *>(&u[0]);
        float v[8];
#pragma unroll
        for (int q = 0; q < 8; ++q) v[q] = f[q];
        return mx_quantize8_f32(v, scale);
    }
}

template <int DT>
__device__ __forceinline__ void from_f32(const float (&v)[8], uint4 (&u)[Elem<DT>::kVec])
{
    if constexpr (DT == MOE_DTYPE_BF16) {
        __nv_bfloat162 *h = reinterpret_cast<__nv_bfloat162 *>(&u[0]);
#pragma unroll
        for (int q = 0; q < 4; ++q) h[q] = __floats2bfloat162_rn(v[2 * q], v[2 * q + 1]);
    } else if constexpr (DT == MOE_DTYPE_F16) {
        __half2 *h = reinterpret_cast<__half2 *>(&u[0]);
#pragma unroll
        for (int q = 0; q < 4; ++q) h[q] = __floats2half2_rn(v[2 * q], v[2 * q + 1]);
    } else {
        float *f = reinterpret_cast<float *>(&u[0]);
#pragma unroll
        for (int q = 0; q < 8; ++q) f[q] = v[q];
    }
}

struct RowParams {
    char *x;             // rows of `stride` bytes
    long long stride;
    uint8_t *codes;      // [rows, cols/2], of 8 bits [rows, cols]
    uint8_t *scales;     // [rows, pitch]
    long long units;     // rows * cols/8
    int upr;             // units per row
    unsigned magic;      // n / upr = (n * magic >> 32) >> shift for n < 2^31
    int shift;
    int pitch;
};

// The CTA's first unit as (row, unit in the row), by one 64-bit division; a thread's own units then take a
// multiplication each (a division each made bf16 rows instruction bound: 255 us for 65536 x 7168).
struct UnitBase { long long row; unsigned col; };

__device__ __forceinline__ UnitBase unit_base(const RowParams &p, long long first)
{
    UnitBase b;
    b.row = first / p.upr;
    b.col = (unsigned)(first - b.row * p.upr);
    return b;
}

__device__ __forceinline__ void store_scale(const RowParams &p, long long row, unsigned block, uint32_t s)
{
    uint8_t *dst = p.scales + row * p.pitch;
    dst[block] = (uint8_t)s;
    if ((int)block * 4 + 4 == p.upr)                          // the row's last block also clears the padding
        for (int q = p.upr / 4; q < p.pitch; ++q) dst[q] = 0;
}

// Large calls: a warp takes 128 units (32 blocks), four per lane, and trades code words within its quads of lanes
// so that a lane stores the 16 bytes and the scale of one block.
template <int DT>
__global__ void __launch_bounds__(kRowThreads) k_mx_quantize(RowParams p)
{
    const long long first = (long long)blockIdx.x * (kRowThreads * 4);
    const UnitBase b = unit_base(p, first);
    const int lane = threadIdx.x & 31, w0 = (threadIdx.x >> 5) * 128;
    uint4 in[4][Elem<DT>::kVec];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const unsigned u = w0 + 32 * i + lane, off = b.col + u;
        const unsigned dr = __umulhi(off, p.magic) >> p.shift;
        const uint4 *src = reinterpret_cast<const uint4 *>(p.x + (b.row + dr) * p.stride) + (size_t)(off - dr * p.upr) * Elem<DT>::kVec;
#pragma unroll
        for (int q = 0; q < Elem<DT>::kVec; ++q) in[i][q] = first + u < p.units ? __ldg(src + q) : make_uint4(0u, 0u, 0u, 0u);
    }
    uint32_t w[4], s[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = quantize8<DT>(in[i], s[i]);
    const uint32_t scale = mx_transpose(w, s, lane);
    const unsigned u = w0 + 4 * mx_block_of_lane(lane), off = b.col + u;     // first unit of this lane's block
    if (first + u < p.units) {
        reinterpret_cast<uint4 *>(p.codes)[(first + u) >> 2] = make_uint4(w[0], w[1], w[2], w[3]);
        const unsigned dr = __umulhi(off, p.magic) >> p.shift;
        store_scale(p, b.row + dr, (off - dr * p.upr) >> 2, scale);
    }
}

// Small calls: a unit per thread, so that there are as many CTAs as possible.
template <int DT>
__global__ void __launch_bounds__(kRowThreads) k_mx_quantize_small(RowParams p)
{
    const long long first = (long long)blockIdx.x * kRowThreads, u = first + threadIdx.x;
    const UnitBase b = unit_base(p, first);
    const unsigned off = b.col + threadIdx.x;
    const unsigned dr = __umulhi(off, p.magic) >> p.shift;
    const unsigned col = off - dr * p.upr;
    const uint4 *src = reinterpret_cast<const uint4 *>(p.x + (b.row + dr) * p.stride) + (size_t)col * Elem<DT>::kVec;
    uint4 in[Elem<DT>::kVec];
#pragma unroll
    for (int q = 0; q < Elem<DT>::kVec; ++q) in[q] = u < p.units ? __ldg(src + q) : make_uint4(0u, 0u, 0u, 0u);
    uint32_t s;
    const uint32_t c = quantize8<DT>(in, s);
    if (u < p.units) {
        reinterpret_cast<uint32_t *>(p.codes)[u] = c;
        if ((col & 3u) == 0u) store_scale(p, b.row + dr, col >> 2, s);
    }
}

// The codes of a unit of eight elements and their values.
template <int BITS> struct Codes;
template <> struct Codes<4> { typedef uint32_t Word; };
template <> struct Codes<8> { typedef uint2 Word; };
__device__ __forceinline__ void unpack8(uint32_t c, float (&v)[8]) { mx_unpack8(c, v); }
__device__ __forceinline__ void unpack8(uint2 c, float (&v)[8]) { mx8_unpack4(c.x, v); mx8_unpack4(c.y, v + 4); }

template <int DT, int UN, int BITS>
__global__ void __launch_bounds__(kRowThreads) k_mx_dequantize(RowParams p)
{
    typedef typename Codes<BITS>::Word Word;
    const long long first = (long long)blockIdx.x * (kRowThreads * UN);
    const UnitBase b = unit_base(p, first);
    Word c[UN];
    uint32_t s[UN];
    long long row[UN]; unsigned col[UN];
#pragma unroll
    for (int i = 0; i < UN; ++i) {
        const unsigned off = b.col + i * kRowThreads + threadIdx.x;
        const unsigned dr = __umulhi(off, p.magic) >> p.shift;
        row[i] = b.row + dr; col[i] = off - dr * p.upr;
        const long long u = first + i * kRowThreads + threadIdx.x;
        if (u < p.units) {
            c[i] = __ldg(reinterpret_cast<const Word *>(p.codes) + u);
            s[i] = __ldg(p.scales + row[i] * p.pitch + (col[i] >> 2));
        }
    }
#pragma unroll
    for (int i = 0; i < UN; ++i) {
        if (first + i * kRowThreads + threadIdx.x >= p.units) continue;
        float v[8];
        unpack8(c[i], v);
        const float scale = mx_scale_value(s[i]);
#pragma unroll
        for (int q = 0; q < 8; ++q) v[q] *= scale;            // exact unless the type's range is left
        uint4 o[Elem<DT>::kVec];
        from_f32<DT>(v, o);
        uint4 *dst = reinterpret_cast<uint4 *>(p.x + row[i] * p.stride) + (size_t)col[i] * Elem<DT>::kVec;
#pragma unroll
        for (int q = 0; q < Elem<DT>::kVec; ++q) dst[q] = o[q];
    }
}

bool aligned(const void *p, unsigned a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

// Checks shared by both directions; fills everything but the launch shape.
moe_status fill(RowParams *p, const void *x, int32_t dtype, long long rows, int32_t cols, long long row_stride,
                const uint8_t *codes, const uint8_t *scales, int bits = 4)
{
    if (rows < 0 || cols < kMxBlock || cols % kMxBlock != 0) return MOE_ERR_INVALID_ARG;
    if (dtype != MOE_DTYPE_BF16 && dtype != MOE_DTYPE_F16 && dtype != MOE_DTYPE_F32) return MOE_ERR_INVALID_ARG;
    const int size = dtype == MOE_DTYPE_F32 ? 4 : 2;
    if (rows > 1 && row_stride < cols) return MOE_ERR_INVALID_ARG;
    if (rows > (1ll << 40) / cols) return MOE_ERR_CAPACITY;          // 2^40 elements
    if (row_stride > (1ll << 40)) return MOE_ERR_INVALID_ARG;
    p->units = rows * (cols / 8);
    if (rows == 0) return MOE_OK;
    if (!x || !codes || !scales || !aligned(x, 16) || !aligned(codes, 16) || !aligned(scales, 16)) return MOE_ERR_INVALID_ARG;
    if (rows > 1 && (row_stride * size) % 16 != 0) return MOE_ERR_INVALID_ARG;
    // One side is read while the other is written, in no particular order.
    const size_t row_bytes = (size_t)cols * size, code_bytes = (size_t)rows * cols * bits / 8, stride_bytes = rows > 1 ? (size_t)row_stride * size : row_bytes;
    if (rows_overlap(x, rows, row_bytes, stride_bytes, codes, code_bytes) ||
        rows_overlap(x, rows, row_bytes, stride_bytes, scales, (size_t)rows * mx_scale_pitch(cols)) ||
        ranges_overlap(codes, code_bytes, scales, (size_t)rows * mx_scale_pitch(cols)))
        return MOE_ERR_INVALID_ARG;
    p->x = static_cast<char *>(const_cast<void *>(x));
    p->stride = row_stride * size;
    p->codes = const_cast<uint8_t *>(codes);
    p->scales = const_cast<uint8_t *>(scales);
    p->upr = cols / 8;
    // With 2^l >= upr, magic = ceil(2^(31 + l) / upr) is below 2^32 and exact for n < 2^31: the quotient is too large
    // by n * (magic * upr - 2^(31 + l)) / (upr * 2^(31 + l)) < 1 / upr at most.
    int l = 0;
    while ((1ll << l) < p->upr) ++l;
    p->magic = (unsigned)(((1ull << (31 + l)) + p->upr - 1) / p->upr);
    p->shift = l - 1;
    p->pitch = mx_scale_pitch(cols);
    return MOE_OK;
}

// Four units per thread keep enough bytes in flight to fill HBM; a call too small to give every SM a
// CTA of four-unit threads is spread over four times as many CTAs instead (one unit per thread).
constexpr long long kFewUnits = 148ll * 4 * kRowThreads;

template <int DT>
void launch_quantize(const RowParams &p, cudaStream_t st)
{
    if (p.units <= kFewUnits)
        k_mx_quantize_small<DT><<<(unsigned)((p.units + kRowThreads - 1) / kRowThreads), kRowThreads, 0, st>>>(p);
    else
        k_mx_quantize<DT><<<(unsigned)((p.units + 4 * kRowThreads - 1) / (4 * kRowThreads)), kRowThreads, 0, st>>>(p);
}

template <int DT, int BITS>
void launch_dequantize(const RowParams &p, cudaStream_t st)
{
    if (p.units <= kFewUnits)
        k_mx_dequantize<DT, 1, BITS><<<(unsigned)((p.units + kRowThreads - 1) / kRowThreads), kRowThreads, 0, st>>>(p);
    else
        k_mx_dequantize<DT, 4, BITS><<<(unsigned)((p.units + 4 * kRowThreads - 1) / (4 * kRowThreads)), kRowThreads, 0, st>>>(p);
}

template <int BITS>
moe_status dequantize(const uint8_t *codes, const uint8_t *scales, int64_t rows, int32_t cols, void *y, int32_t dtype, int64_t row_stride,
                      void *cuda_stream)
{
    RowParams p;
    const moe_status ms = fill(&p, y, dtype, rows, cols, row_stride, codes, scales, BITS);
    if (ms != MOE_OK || p.units == 0) return ms;
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    if (dtype == MOE_DTYPE_BF16) launch_dequantize<MOE_DTYPE_BF16, BITS>(p, st);
    else if (dtype == MOE_DTYPE_F16) launch_dequantize<MOE_DTYPE_F16, BITS>(p, st);
    else launch_dequantize<MOE_DTYPE_F32, BITS>(p, st);
    return cudaGetLastError() == cudaSuccess ? MOE_OK : MOE_ERR_CUDA;
}

}  // namespace

extern "C" {

int32_t moe_mx_scale_pitch(int32_t cols)
{
    return cols < kMxBlock || cols % kMxBlock != 0 ? 0 : mx_scale_pitch(cols);
}

moe_status moe_mx_quantize(const void *x, int32_t dtype, int64_t rows, int32_t cols, int64_t row_stride, uint8_t *codes,
                           uint8_t *scales, void *cuda_stream)
{
    RowParams p;
    const moe_status ms = fill(&p, x, dtype, rows, cols, row_stride, codes, scales);
    if (ms != MOE_OK || p.units == 0) return ms;
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    if (dtype == MOE_DTYPE_BF16) launch_quantize<MOE_DTYPE_BF16>(p, st);
    else if (dtype == MOE_DTYPE_F16) launch_quantize<MOE_DTYPE_F16>(p, st);
    else launch_quantize<MOE_DTYPE_F32>(p, st);
    return cudaGetLastError() == cudaSuccess ? MOE_OK : MOE_ERR_CUDA;
}

moe_status moe_mx_dequantize(const uint8_t *codes, const uint8_t *scales, int64_t rows, int32_t cols, void *y, int32_t dtype,
                             int64_t row_stride, void *cuda_stream)
{
    return dequantize<4>(codes, scales, rows, cols, y, dtype, row_stride, cuda_stream);
}

moe_status moe_kept_dequantize(const uint8_t *codes, const uint8_t *scales, int64_t rows, int32_t cols, void *y, int32_t dtype,
                              int64_t row_stride, void *cuda_stream)
{
    return dequantize<8>(codes, scales, rows, cols, y, dtype, row_stride, cuda_stream);
}

}  // extern "C"
