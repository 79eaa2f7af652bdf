// moe_rms_norm / moe_rms_norm_backward: the norm in front of a layer, with the residual's addition, and its gradient.
//
//   h = x + residual (rounded to the rows' type), rstd = 1 / sqrt(mean(h^2) + eps), y = h * rstd * weight,
//   and y in 8 bits (mx8_format.cuh) where it is kept for a backward pass
//   backward, with n = h * rstd and g = dy * weight:  dx = rstd * (g - n * mean(g * n)) + dh,  d_weight = sum over rows of dy * n
//
// Both are one pass over the rows and bound by HBM.  A row is taken by a warp up to 1024 columns, by a CTA above, with as many
// warps as make four units a thread (a fixed 256 threads lost half of the bandwidth at 1536 columns).  A thread owns units of eight
// consecutive elements (one 16-byte access of a 16-bit type), so four neighbouring lanes own a block of the 8-bit form.  The forward pass holds a row in registers between the reduction and the
// result and has a CTA per row.  The backward pass has as many CTAs as fit, because each also sums d_weight over its rows; its
// next rows are on their way to shared memory meanwhile (k_rms_norm_backward_ring).  All sums are fp32, in an order that
// depends on the sizes alone; every output is rounded once.
#include "../../include/moe_route.h"

#include <algorithm>
#include <mutex>
#include <type_traits>

#include "mx8_format.cuh"

namespace {

using namespace moe;

constexpr int kUnits = 4;                  // units of eight elements per thread
constexpr int kMaxThreads = 512;           // of a CTA that has a row
constexpr int kMaxCols = kMaxThreads * kUnits * 8;
constexpr int kSms = 148;
constexpr int kRingBytes = 220 * 1024;     // shared memory of an SM for the rows of a backward pass

template <int DT> constexpr int kVec = DT == MOE_DTYPE_F32 ? 2 : 1;   // 16-byte words of a unit

// Rows are read once.  (Not through the read-only path: an output may take the place of an input.)
__device__ __forceinline__ uint4 load_v4(const uint4 *p)
{
    uint4 v;
    asm volatile("ld.global.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p) : "memory");
    return v;
}

template <int DT>
__device__ __forceinline__ void to_f32(const uint4 (&u)[kVec<DT>], float (&v)[8])
{
    if constexpr (DT == MOE_DTYPE_F32) {
        const uint32_t w[8] = {u[0].x, u[0].y, u[0].z, u[0].w, u[1].x, u[1].y, u[1].z, u[1].w};
#pragma unroll
        for (int q = 0; q < 8; ++q) v[q] = __uint_as_float(w[q]);
    } else {
        const uint32_t w[4] = {u[0].x, u[0].y, u[0].z, u[0].w};
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            if constexpr (DT == MOE_DTYPE_BF16) {
                v[2 * q] = __uint_as_float(w[q] << 16);
                v[2 * q + 1] = __uint_as_float(w[q] & 0xffff0000u);
            } else {
                const float2 f = __half22float2(*reinterpret_cast<const __half2 *>(&w[q]));
                v[2 * q] = f.x; v[2 * q + 1] = f.y;
            }
        }
    }
}

template <int DT>
__device__ __forceinline__ void from_f32(const float (&v)[8], uint4 (&u)[kVec<DT>])
{
    uint32_t *w = reinterpret_cast<uint32_t *>(&u[0]);
    if constexpr (DT == MOE_DTYPE_F32) {
#pragma unroll
        for (int q = 0; q < 8; ++q) w[q] = __float_as_uint(v[q]);
    } else {
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            if constexpr (DT == MOE_DTYPE_BF16) {
                const __nv_bfloat162 h = __floats2bfloat162_rn(v[2 * q], v[2 * q + 1]);
                w[q] = *reinterpret_cast<const uint32_t *>(&h);
            } else {
                const __half2 h = __floats2half2_rn(v[2 * q], v[2 * q + 1]);
                w[q] = *reinterpret_cast<const uint32_t *>(&h);
            }
        }
    }
}

// Eight elements of the weight, of any of the types.
__device__ __forceinline__ void weight8(const void *weight, int dtype, int unit, float (&v)[8])
{
    const uint4 *src = static_cast<const uint4 *>(weight);
    if (dtype == MOE_DTYPE_F32) {
        const uint4 u[2] = {__ldg(src + 2 * unit), __ldg(src + 2 * unit + 1)};
        to_f32<MOE_DTYPE_F32>(u, v);
    } else {
        const uint4 u[1] = {__ldg(src + unit)};
        if (dtype == MOE_DTYPE_BF16) to_f32<MOE_DTYPE_BF16>(u, v);
        else to_f32<MOE_DTYPE_F16>(u, v);
    }
}

__device__ __forceinline__ float warp_sum(float v)
{
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) v += __shfl_xor_sync(0xffffffffu, v, off);
    return v;
}

// Sum over the CTA; `scratch` holds two sets of a float per warp, which calls take in turn.
__device__ __forceinline__ float cta_sum(float v, float *scratch, int turn)
{
    const int lane = threadIdx.x & 31;
    v = warp_sum(v);
    scratch += turn * (kMaxThreads / 32);
    if (lane == 0) scratch[threadIdx.x >> 5] = v;
    __syncthreads();
    return warp_sum(lane < (int)blockDim.x / 32 ? scratch[lane] : 0.0f);
}

struct NormParams {
    const uint4 *x, *residual;     // rows of x_stride and r_stride words of 16 bytes; residual may be NULL
    long long x_stride, r_stride;
    const void *weight;
    int weight_dtype;
    float eps;
    long long rows;
    int units;                     // of a row
    uint4 *h, *y;                  // h may be NULL
    float *rstd;                   // may be NULL
    uint8_t *codes, *scales;       // may be NULL
    int pitch;
};

// UN units per thread; WARP: eight rows to a CTA, a warp each, and not one to the CTA.
template <int DT, int UN, bool WARP>
__global__ void __launch_bounds__(WARP ? 256 : kMaxThreads) k_rms_norm(NormParams p)
{
    constexpr int V = kVec<DT>;
    __shared__ float scratch[2 * kMaxThreads / 32];
    const int tid = WARP ? threadIdx.x & 31 : threadIdx.x, threads = WARP ? 32 : blockDim.x;
    const long long row = WARP ? (long long)blockIdx.x * 8 + (threadIdx.x >> 5) : blockIdx.x;
    if (WARP && row >= p.rows) return;
    const uint4 *x = p.x + row * p.x_stride, *res = p.residual ? p.residual + row * p.r_stride : nullptr;
    uint4 in[UN][V], add[UN][V];
#pragma unroll
    for (int i = 0; i < UN; ++i) {
        const int u = i * threads + tid;
#pragma unroll
        for (int q = 0; q < V; ++q) {
            in[i][q] = u < p.units ? load_v4(x + u * V + q) : make_uint4(0u, 0u, 0u, 0u);
            if (res) add[i][q] = u < p.units ? load_v4(res + u * V + q) : make_uint4(0u, 0u, 0u, 0u);
        }
    }
    float sum = 0.0f;
#pragma unroll
    for (int i = 0; i < UN; ++i) {
        float a[8];
        to_f32<DT>(in[i], a);
        if (res) {
            float b[8];
            to_f32<DT>(add[i], b);
#pragma unroll
            for (int q = 0; q < 8; ++q) a[q] += b[q];
            from_f32<DT>(a, in[i]);                            // the norm is that of the stored sum
            to_f32<DT>(in[i], a);
        }
#pragma unroll
        for (int q = 0; q < 8; ++q) sum += a[q] * a[q];
        const int u = i * threads + tid;
        if (p.h && u < p.units)
#pragma unroll
            for (int q = 0; q < V; ++q) p.h[(row * p.units + u) * V + q] = in[i][q];
    }
    const float rstd = rsqrtf((WARP ? warp_sum(sum) : cta_sum(sum, scratch, 0)) / (float)(p.units * 8) + p.eps);
    if (p.rstd && tid == 0) p.rstd[row] = rstd;
#pragma unroll
    for (int i = 0; i < UN; ++i) {
        const int u = i * threads + tid;
        const bool inside = u < p.units;                       // with an 8-bit form whole blocks: all four lanes of one or none
        float a[8], w[8];
        to_f32<DT>(in[i], a);
        if (inside) weight8(p.weight, p.weight_dtype, u, w);
#pragma unroll
        for (int q = 0; q < 8; ++q) a[q] = inside ? a[q] * rstd * w[q] : 0.0f;
        if (inside) {
            uint4 o[V];
            from_f32<DT>(a, o);
#pragma unroll
            for (int q = 0; q < V; ++q) p.y[(row * p.units + u) * V + q] = o[q];
        }
        if (p.codes) {
            uint32_t amax = mx8_amax(a);
            amax = max(amax, __shfl_xor_sync(0xffffffffu, amax, 1));
            amax = max(amax, __shfl_xor_sync(0xffffffffu, amax, 2));
            const uint32_t s = mx8_scale_byte(amax);
            if (inside) *reinterpret_cast<uint2 *>(p.codes + (row * p.units + u) * 8) = mx8_quantize8(a, s);
            if ((u & 3) == 0 && inside) p.scales[row * p.pitch + u / 4] = (uint8_t)s;
        }
    }
    if (p.codes)                                               // the padding of the scales is written as 0
        for (int b = p.units / 4 + tid; b < p.pitch; b += threads) p.scales[row * p.pitch + b] = 0;
}

struct NormBackwardParams {
    const uint4 *dy, *dh, *h;      // dh may be NULL
    const float *rstd;
    const void *weight;
    int weight_dtype;
    long long rows;
    int units;
    uint4 *dx;
    float *partial;                // [CTAs, cols]
};

// Two fp32 in one 64-bit register: sm_100 multiplies and adds them with one instruction, rounded as two.
typedef unsigned long long Pair;

__device__ __forceinline__ Pair pair(float a, float b)
{
    Pair r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
    return r;
}

__device__ __forceinline__ void split(Pair p, float &a, float &b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(p)); }

__device__ __forceinline__ Pair mul2(Pair a, Pair b)
{
    Pair r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}

__device__ __forceinline__ Pair fma2(Pair a, Pair b, Pair c)
{
    Pair r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}

template <int DT>
__device__ __forceinline__ void to_pairs(const uint4 (&u)[kVec<DT>], Pair (&v)[4])
{
    float f[8];
    to_f32<DT>(u, f);
#pragma unroll
    for (int q = 0; q < 4; ++q) v[q] = pair(f[2 * q], f[2 * q + 1]);
}

__device__ __forceinline__ void weight_pairs(const NormBackwardParams &p, int unit, Pair (&w)[4])
{
    float f[8];
    weight8(p.weight, p.weight_dtype, unit, f);
#pragma unroll
    for (int q = 0; q < 4; ++q) w[q] = pair(f[2 * q], f[2 * q + 1]);
}

// A unit of a row: n = h * rstd, and what the row's mean and d_weight take from it.
__device__ __forceinline__ void norm_sums(const Pair (&dy)[4], const Pair (&h)[4], const Pair (&w)[4], Pair rstd, Pair &sum, Pair (&acc)[4])
{
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        const Pair n = mul2(h[q], rstd);
        sum = fma2(mul2(dy[q], w[q]), n, sum);
        acc[q] = fma2(dy[q], n, acc[q]);
    }
}

// rstd * (dy * w - n * mean) + past, in the rows' type
template <int DT>
__device__ __forceinline__ void norm_gradient(const Pair (&dy)[4], const Pair (&h)[4], const Pair (&w)[4], Pair rstd, Pair minus_mean,
                                              const Pair (&past)[4], uint4 (&out)[kVec<DT>])
{
    float d[8];
#pragma unroll
    for (int q = 0; q < 4; ++q)
        split(fma2(fma2(mul2(h[q], rstd), minus_mean, mul2(dy[q], w[q])), rstd, past[q]), d[2 * q], d[2 * q + 1]);
    from_f32<DT>(d, out);
}

__device__ __forceinline__ float sum_of(Pair p)
{
    float a, b;
    split(p, a, b);
    return a + b;
}

__device__ __forceinline__ void store_sums(float *dst, const Pair (&acc)[4])
{
#pragma unroll
    for (int q = 0; q < 4; q += 2) {
        float4 v;
        split(acc[q], v.x, v.y); split(acc[q + 1], v.z, v.w);
        reinterpret_cast<float4 *>(dst)[q / 2] = v;
    }
}

// Rows of up to 1024 columns: a warp each, eight to a CTA, whose sums of d_weight meet in shared memory.
template <int DT, int UN>
__global__ void __launch_bounds__(256) k_rms_norm_backward(NormBackwardParams p)
{
    constexpr int V = kVec<DT>, kRows = 8;
    extern __shared__ float sums[];                            // [kRows, cols]
    const int lane = threadIdx.x & 31, sub = threadIdx.x >> 5;
    Pair acc[UN][4] = {}, w[UN][4] = {};                       // two +0 are 64 bits of zero
#pragma unroll
    for (int i = 0; i < UN; ++i)
        if (i * 32 + lane < p.units) weight_pairs(p, i * 32 + lane, w[i]);
    for (long long row = (long long)blockIdx.x * kRows + sub; row < p.rows; row += (long long)gridDim.x * kRows) {
        uint4 a[UN][V], b[UN][V], c[UN][V];
#pragma unroll
        for (int i = 0; i < UN; ++i) {
            const int u = i * 32 + lane;
#pragma unroll
            for (int q = 0; q < V; ++q) {
                const long long at = (row * p.units + u) * V + q;
                a[i][q] = b[i][q] = c[i][q] = make_uint4(0u, 0u, 0u, 0u);
                if (u < p.units) {
                    a[i][q] = load_v4(p.dy + at);
                    b[i][q] = load_v4(p.h + at);
                    if (p.dh) c[i][q] = load_v4(p.dh + at);
                }
            }
        }
        const float r = __ldg(p.rstd + row);
        const Pair rstd = pair(r, r);
        Pair sum = 0;
#pragma unroll
        for (int i = 0; i < UN; ++i) {
            Pair dy[4], h[4];
            to_pairs<DT>(a[i], dy); to_pairs<DT>(b[i], h);
            norm_sums(dy, h, w[i], rstd, sum, acc[i]);
        }
        const float mean = warp_sum(sum_of(sum)) / (float)(p.units * 8);
        const Pair minus_mean = pair(-mean, -mean);
#pragma unroll
        for (int i = 0; i < UN; ++i) {
            const int u = i * 32 + lane;
            if (u >= p.units) continue;
            Pair dy[4], h[4], past[4];
            to_pairs<DT>(a[i], dy); to_pairs<DT>(b[i], h); to_pairs<DT>(c[i], past);
            uint4 o[V];
            norm_gradient<DT>(dy, h, w[i], rstd, minus_mean, past, o);
#pragma unroll
            for (int q = 0; q < V; ++q) p.dx[(row * p.units + u) * V + q] = o[q];
        }
    }
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const int cols = p.units * 8;
#pragma unroll
    for (int i = 0; i < UN; ++i)
        if (i * 32 + lane < p.units) store_sums(sums + sub * cols + (i * 32 + lane) * 8, acc[i]);
    __syncthreads();
    for (int c = threadIdx.x; c < cols; c += 256) {
        float s = 0.0f;
#pragma unroll
        for (int r = 0; r < kRows; ++r) s += sums[r * cols + c];
        p.partial[(size_t)blockIdx.x * cols + c] = s;
    }
}

// Longer rows: a CTA each.  Its rows of dy, h and dh come by asynchronous copies, STAGES - 1 rows ahead, into a ring in shared
// memory; every thread reads back what it copied itself, so a wait for its own copies is all that a stage takes.  (With
// loads to registers and two CTAs per SM: 254 us for 16384 x 7168 in bf16, whose bytes take 143.)
template <int DT, int STAGES>
__global__ void __launch_bounds__(kMaxThreads) k_rms_norm_backward_ring(NormBackwardParams p)
{
    constexpr int V = kVec<DT>;
    __shared__ float scratch[2 * kMaxThreads / 32];
    extern __shared__ uint4 ring[];                            // [STAGES][dy, h, dh][units * V]
    const int tid = threadIdx.x, threads = blockDim.x, words = p.units * V, tensors = p.dh ? 3 : 2;
    Pair acc[kUnits][4] = {}, w[kUnits][4] = {};               // two +0 are 64 bits of zero
#pragma unroll
    for (int i = 0; i < kUnits; ++i)
        if (i * threads + tid < p.units) weight_pairs(p, i * threads + tid, w[i]);
    const auto ask = [&](long long row, uint4 *stage) {
        if (row < p.rows)
#pragma unroll
            for (int i = 0; i < kUnits; ++i) {
                const int u = i * threads + tid;
                if (u >= p.units) continue;
#pragma unroll
                for (int q = 0; q < V; ++q) {
                    const long long at = row * words + u * V + q;
                    cp_async_16(stage + u * V + q, p.dy + at);
                    cp_async_16(stage + words + u * V + q, p.h + at);
                    if (tensors == 3) cp_async_16(stage + 2 * words + u * V + q, p.dh + at);
                }
            }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
    const long long step = gridDim.x;
    const int stage_words = tensors * words;
    int fill = 0, take = 0, turn = 0;
#pragma unroll
    for (int s = 0; s < STAGES - 1; ++s) ask(blockIdx.x + s * step, ring + s * stage_words);
    fill = (STAGES - 1) * stage_words;
    for (long long row = blockIdx.x; row < p.rows; row += step) {
        ask(row + (STAGES - 1) * step, ring + fill);
        fill = fill == (STAGES - 1) * stage_words ? 0 : fill + stage_words;
        const float r = __ldg(p.rstd + row);
        const Pair rstd = pair(r, r);
        asm volatile("cp.async.wait_group %0;" ::"n"(STAGES - 1) : "memory");
        const uint4 *in = ring + take;
        take = take == (STAGES - 1) * stage_words ? 0 : take + stage_words;
        Pair sum = 0;
#pragma unroll
        for (int i = 0; i < kUnits; ++i) {
            const int u = i * threads + tid;
            if (u >= p.units) continue;
            uint4 a[V], b[V];
#pragma unroll
            for (int q = 0; q < V; ++q) { a[q] = in[u * V + q]; b[q] = in[words + u * V + q]; }
            Pair dy[4], h[4];
            to_pairs<DT>(a, dy); to_pairs<DT>(b, h);
            norm_sums(dy, h, w[i], rstd, sum, acc[i]);
        }
        const float mean = cta_sum(sum_of(sum), scratch, turn) / (float)(p.units * 8);
        const Pair minus_mean = pair(-mean, -mean);
        turn ^= 1;
#pragma unroll
        for (int i = 0; i < kUnits; ++i) {
            const int u = i * threads + tid;
            if (u >= p.units) continue;
            uint4 a[V], b[V], c[V];
#pragma unroll
            for (int q = 0; q < V; ++q) {
                a[q] = in[u * V + q]; b[q] = in[words + u * V + q];
                c[q] = tensors == 3 ? in[2 * words + u * V + q] : make_uint4(0u, 0u, 0u, 0u);
            }
            Pair dy[4], h[4], past[4];
            to_pairs<DT>(a, dy); to_pairs<DT>(b, h); to_pairs<DT>(c, past);
            uint4 o[V];
            norm_gradient<DT>(dy, h, w[i], rstd, minus_mean, past, o);
#pragma unroll
            for (int q = 0; q < V; ++q) p.dx[row * words + u * V + q] = o[q];
        }
    }
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
#pragma unroll
    for (int i = 0; i < kUnits; ++i)
        if (i * threads + tid < p.units) store_sums(p.partial + ((size_t)blockIdx.x * p.units + i * threads + tid) * 8, acc[i]);
}

// d_weight: the CTAs' sums added up, 64 of them side by side for each four columns (two in a warp, whose loads are lines).
constexpr int kWeightQuads = 16;           // of a CTA
__global__ void __launch_bounds__(1024) k_norm_weight(const float4 *partial, int ctas, int quads, float4 *d_weight)
{
    __shared__ float4 sums[32][kWeightQuads];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, c = blockIdx.x * kWeightQuads + (lane & 15);
    asm volatile("griddepcontrol.wait;" ::: "memory");         // launched while the rows' kernel drains
    float4 s = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    if (c < quads) {
#pragma unroll 4
        for (int i = 2 * warp + (lane >> 4); i < ctas; i += 64) {
            const float4 v = __ldcg(partial + (size_t)i * quads + c);
            s.x += v.x; s.y += v.y; s.z += v.z; s.w += v.w;
        }
    }
    s.x += __shfl_down_sync(0xffffffffu, s.x, 16); s.y += __shfl_down_sync(0xffffffffu, s.y, 16);
    s.z += __shfl_down_sync(0xffffffffu, s.z, 16); s.w += __shfl_down_sync(0xffffffffu, s.w, 16);
    if (lane < 16) sums[warp][lane] = s;
    __syncthreads();
    if (threadIdx.x >= kWeightQuads || c >= quads) return;
#pragma unroll 8
    for (int i = 1; i < 32; ++i) {
        const float4 v = sums[i][lane];
        s.x += v.x; s.y += v.y; s.z += v.z; s.w += v.w;
    }
    d_weight[c] = s;
}

bool aligned(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

bool is_dtype(int32_t d) { return d == MOE_DTYPE_BF16 || d == MOE_DTYPE_F16 || d == MOE_DTYPE_F32; }

// f(type, units per thread, whether a row is a warp's) for the kernel that rows of `units` units of this type take
template <typename F>
void with_kernel(int32_t dtype, int units, F f)
{
    using std::integral_constant;
    const auto by_width = [&](auto dt) {
        if (units <= 32) f(dt, integral_constant<int, 1>(), std::true_type());
        else if (units <= 64) f(dt, integral_constant<int, 2>(), std::true_type());
        else if (units <= 32 * kUnits) f(dt, integral_constant<int, kUnits>(), std::true_type());
        else f(dt, integral_constant<int, kUnits>(), std::false_type());
    };
    if (dtype == MOE_DTYPE_BF16) by_width(integral_constant<int, MOE_DTYPE_BF16>());
    else if (dtype == MOE_DTYPE_F16) by_width(integral_constant<int, MOE_DTYPE_F16>());
    else by_width(integral_constant<int, MOE_DTYPE_F32>());
}

// Threads of the CTA that takes a row.
int row_threads(int units) { return (units + 32 * kUnits - 1) / (32 * kUnits) * 32; }

// CTAs of a backward pass at most, each with a row of partial sums of d_weight: 512 threads of CTAs with a row (their
// registers fill an SM), two CTAs of eight warps with a row each.
int64_t backward_ctas(int64_t rows, int units)
{
    if (units <= 32 * kUnits) return std::min<int64_t>((rows + 7) / 8, 2 * kSms);
    // but not for fewer than four rows where one CTA an SM has as many: their sums are written and read again
    const int64_t most = std::min(8, kMaxThreads / row_threads(units)) * kSms, few = std::max(std::min<int64_t>(rows, kSms), (rows + 3) / 4);
    return std::min(most, few);
}

// A function's attributes are those of one device: set at its first use there.
template <int DT, int STAGES>
cudaError_t allow_ring()
{
    constexpr int kDevices = 64;
    static std::once_flag once[kDevices];
    static cudaError_t attr[kDevices];
    int device;
    const cudaError_t e = cudaGetDevice(&device);
    if (e != cudaSuccess) return e;
    if (device >= kDevices) return cudaErrorInvalidDevice;
    std::call_once(once[device], [&] { attr[device] = cudaFuncSetAttribute(k_rms_norm_backward_ring<DT, STAGES>, cudaFuncAttributeMaxDynamicSharedMemorySize, kRingBytes); });
    return attr[device];
}

moe_status check_norm(int32_t dtype, int32_t weight_dtype, int64_t rows, int32_t cols)
{
    if (rows < 0 || cols < 8 || cols % 8 != 0 || cols > kMaxCols || !is_dtype(dtype) || !is_dtype(weight_dtype)) return MOE_ERR_INVALID_ARG;
    return rows > (1ll << 31) - 1 ? MOE_ERR_CAPACITY : MOE_OK;
}

}  // namespace

extern "C" {

moe_status moe_rms_norm(const void *x, int64_t x_stride, const void *residual, int64_t residual_stride, int32_t dtype, int64_t rows,
                        int32_t cols, const void *weight, int32_t weight_dtype, float eps, void *h, void *y, float *rstd, uint8_t *codes,
                        uint8_t *scales, void *cuda_stream)
{
    const moe_status ms = check_norm(dtype, weight_dtype, rows, cols);
    if (ms != MOE_OK) return ms;
    if (!(eps >= 0.0f) || (codes == nullptr) != (scales == nullptr) || (codes && cols % kMxBlock != 0)) return MOE_ERR_INVALID_ARG;
    if (rows == 0) return MOE_OK;
    const long long size = dtype == MOE_DTYPE_F32 ? 4 : 2;
    if (rows > 1 && (x_stride < cols || x_stride > (1ll << 40) || x_stride * size % 16 != 0)) return MOE_ERR_INVALID_ARG;
    if (rows > 1 && residual && (residual_stride < cols || residual_stride > (1ll << 40) || residual_stride * size % 16 != 0))
        return MOE_ERR_INVALID_ARG;
    if (!x || !weight || !y || (residual && !h) || !aligned(x) || !aligned(residual) || !aligned(weight) || !aligned(h) || !aligned(y) ||
        !aligned(codes) || !aligned(scales))
        return MOE_ERR_INVALID_ARG;
    // Outputs may not lie on inputs or on one another, but for h in the place of x or of the residual: a thread
    // has read what it overwrites there.
    const size_t n = rows, row = (size_t)cols * size;
    const struct { const void *at; size_t bytes; } out[5] = {
        {y, n * row}, {codes, codes ? n * cols : 0}, {scales, codes ? n * mx_scale_pitch(cols) : 0}, {rstd, rstd ? n * 4 : 0}, {h, h ? n * row : 0}};
    for (int i = 0; i < 5; ++i) {
        for (int j = 0; j < i; ++j)
            if (ranges_overlap(out[i].at, out[i].bytes, out[j].at, out[j].bytes)) return MOE_ERR_INVALID_ARG;
        if (ranges_overlap(out[i].at, out[i].bytes, weight, (size_t)cols * (weight_dtype == MOE_DTYPE_F32 ? 4 : 2))) return MOE_ERR_INVALID_ARG;
        const bool same_x = i == 4 && h == x && (rows == 1 || x_stride == cols);
        const bool same_r = i == 4 && h == residual && (rows == 1 || residual_stride == cols);
        if (!same_x && rows_overlap(x, rows, row, rows > 1 ? x_stride * size : row, out[i].at, out[i].bytes)) return MOE_ERR_INVALID_ARG;
        if (residual && !same_r && rows_overlap(residual, rows, row, rows > 1 ? residual_stride * size : row, out[i].at, out[i].bytes))
            return MOE_ERR_INVALID_ARG;
    }
    NormParams p;
    p.x = static_cast<const uint4 *>(x); p.residual = static_cast<const uint4 *>(residual);
    p.x_stride = x_stride * size / 16; p.r_stride = residual_stride * size / 16;
    p.weight = weight; p.weight_dtype = weight_dtype; p.eps = eps; p.rows = rows; p.units = cols / 8;
    p.h = static_cast<uint4 *>(h); p.y = static_cast<uint4 *>(y); p.rstd = rstd; p.codes = codes; p.scales = scales;
    p.pitch = mx_scale_pitch(cols);
    with_kernel(dtype, p.units, [&](auto dt, auto un, auto warp) {
        k_rms_norm<dt, un, warp><<<(unsigned)(warp ? (rows + 7) / 8 : rows), warp ? 256 : row_threads(p.units), 0,
                                   static_cast<cudaStream_t>(cuda_stream)>>>(p);
    });
    return cudaGetLastError() == cudaSuccess ? MOE_OK : MOE_ERR_CUDA;
}

size_t moe_rms_norm_backward_workspace(int64_t rows, int32_t cols)
{
    return rows < 1 || cols < 8 || cols % 8 != 0 || cols > kMaxCols ? 0 : (size_t)backward_ctas(rows, cols / 8) * cols * 4;
}

moe_status moe_rms_norm_backward(const void *dy, const void *dh, const void *h, const float *rstd, int32_t dtype, int64_t rows,
                                 int32_t cols, const void *weight, int32_t weight_dtype, void *dx, float *d_weight, void *workspace,
                                 size_t workspace_bytes, void *cuda_stream)
{
    const moe_status ms = check_norm(dtype, weight_dtype, rows, cols);
    if (ms != MOE_OK) return ms;
    if (!d_weight || !aligned(d_weight)) return MOE_ERR_INVALID_ARG;
    cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
    if (rows == 0) return cudaMemsetAsync(d_weight, 0, (size_t)cols * 4, st) == cudaSuccess ? MOE_OK : MOE_ERR_CUDA;
    if (!dy || !h || !rstd || !weight || !dx || !workspace || !aligned(dy) || !aligned(dh) || !aligned(h) || !aligned(weight) || !aligned(dx) ||
        !aligned(workspace))
        return MOE_ERR_INVALID_ARG;
    const size_t need = moe_rms_norm_backward_workspace(rows, cols);
    if (workspace_bytes < need) return MOE_ERR_CAPACITY;
    // dx may take the place of dy, of dh or of h: a thread has read what it overwrites there
    const size_t n = rows, bytes = n * cols * (dtype == MOE_DTYPE_F32 ? 4 : 2), w = (size_t)cols * (weight_dtype == MOE_DTYPE_F32 ? 4 : 2);
    const struct { const void *at; size_t bytes; } out[3] = {{dx, bytes}, {d_weight, (size_t)cols * 4}, {workspace, need}},
        in[5] = {{dy, bytes}, {dh, dh ? bytes : 0}, {h, bytes}, {rstd, n * 4}, {weight, w}};
    for (int i = 0; i < 3; ++i) {
        for (int j = 0; j < i; ++j)
            if (ranges_overlap(out[i].at, out[i].bytes, out[j].at, out[j].bytes)) return MOE_ERR_INVALID_ARG;
        for (int j = 0; j < 5; ++j)
            if (!(i == 0 && j < 3 && dx == in[j].at) && ranges_overlap(out[i].at, out[i].bytes, in[j].at, in[j].bytes)) return MOE_ERR_INVALID_ARG;
    }
    NormBackwardParams p;
    p.dy = static_cast<const uint4 *>(dy); p.dh = static_cast<const uint4 *>(dh); p.h = static_cast<const uint4 *>(h);
    p.rstd = rstd; p.weight = weight; p.weight_dtype = weight_dtype; p.rows = rows; p.units = cols / 8;
    p.dx = static_cast<uint4 *>(dx); p.partial = static_cast<float *>(workspace);
    int ctas = (int)backward_ctas(rows, p.units);
    cudaError_t e = cudaSuccess;
    with_kernel(dtype, p.units, [&](auto dt, auto un, auto warp) {
        if constexpr (warp) {
            k_rms_norm_backward<dt, un><<<ctas, 256, (size_t)8 * cols * 4, st>>>(p);
            e = cudaGetLastError();
        } else {
            // As many CTAs as the registers hold, with two or three rows each in the ring; fewer where not even two fit.  (One CTA
            // of 224 threads with three rows: 255 us for 16384 x 7168 in bf16.)
            const size_t stage = (size_t)cols * (dtype == MOE_DTYPE_F32 ? 4 : 2) * (dh ? 3 : 2);
            int per_sm = std::min(8, kMaxThreads / row_threads(p.units));
            while (per_sm > 1 && kRingBytes / per_sm < 2 * stage) --per_sm;
            const int stages = (int)std::min<size_t>(3, kRingBytes / per_sm / stage);
            ctas = (int)std::min<int64_t>(ctas, per_sm * kSms);
            const auto launch = [&](auto n) {
                e = allow_ring<dt, n>();
                if (e != cudaSuccess) return;
                k_rms_norm_backward_ring<dt, n><<<ctas, row_threads(p.units), stages * stage, st>>>(p);
                e = cudaGetLastError();
            };
            if (stages == 3) launch(std::integral_constant<int, 3>());
            else if (stages == 2) launch(std::integral_constant<int, 2>());
            else launch(std::integral_constant<int, 1>());
        }
    });
    if (e != cudaSuccess) return MOE_ERR_CUDA;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((cols / 4 + kWeightQuads - 1) / kWeightQuads); cfg.blockDim = dim3(1024); cfg.stream = st;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = at; cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, k_norm_weight, static_cast<const float4 *>(workspace), ctas, cols / 4, reinterpret_cast<float4 *>(d_weight)) ==
                   cudaSuccess ? MOE_OK : MOE_ERR_CUDA;
}

}  // extern "C"
