// Gradients of the routed step.
//
// combine:   y[t] = sum_j w[t,j] * scale[slot] * buf[row(t,j)]
//   d_buf[row(t,j)] = bf16(w[t,j] * scale[slot] * dy[t])     (the coefficient is one fp32 multiply, as forward)
//   d_w[t,j]        = scale[slot] * <buf[row(t,j)], dy[t]>    (fp32 sums)
// dispatch:  send[row(t,j)] = x[t];  w[t,:] from the logits of the chosen experts
//   d_x[t]          = bf16(sum_j d_send[row(t,j)])            (k_combine_bulk with coefficients 1)
//   w_j = c * u_j / sum_i u_i with u = exp(l) or u = sigmoid(l), c = route_scale:
//   d_l_j           = w_j * (g_j - sum_i w_i g_i / c) * (1 for softmax, 1 - sigmoid(l_j) = sigmoid(-l_j) for sigmoid)
//   and zero for every expert that was not chosen (the selection itself has no gradient).
#pragma once

#include "combine_kernels.cuh"

namespace moe {

struct CombineBackwardParams {
    const uint4 *buf;            // [T*k, H/8]
    const uint4 *dy;             // [T, H/8]
    uint4 *d_buf;                // [T*k, H/8]
    float *d_weights;            // [T,k]
    int T, k, hv, P;
    const int32_t *dst_row;      // [T*k]
    const float *topk_weights;   // [T,k]
    const int32_t *topk_slot;    // [T,k]
    const float *slot_scale;     // [P]
};

constexpr int kCombineBwdThreads = 256;
constexpr int kCombineBwdUnits = 4;      // 16-byte units of dy a thread keeps in registers
constexpr int kMaxTopKDevice = 16;

// One CTA per token: its threads hold the token's dy row (up to 8192 columns at a time) in registers
// while the k expert rows stream past, each read once for the dot product with the d_buf row going
// out in its place.  Bound by HBM: (1 + 2k) rows of traffic per token.  The next row's loads are
// issued before the present row is worked on.  Dot products are reduced in a fixed order.
__global__ void __launch_bounds__(kCombineBwdThreads) k_combine_backward(CombineBackwardParams p)
{
    constexpr int U = kCombineBwdUnits;
    __shared__ float s_coef[kMaxTopKDevice], s_scale[kMaxTopKDevice];
    __shared__ int s_row[kMaxTopKDevice];
    __shared__ float s_dot[kCombineBwdThreads / 32][kMaxTopKDevice];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, nw = blockDim.x >> 5;
    const int k = p.k;
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    for (int t = blockIdx.x; t < p.T; t += gridDim.x) {
        __syncthreads();                                      // the previous token's tables are free
        if (tid < k) {
            const size_t i = (size_t)t * k + tid;
            const int slot = __ldg(p.topk_slot + i), r = __ldg(p.dst_row + i);
            const bool placed = (unsigned)slot < (unsigned)p.P && r >= 0 && r < (long long)p.T * k;
            const float scale = placed ? __ldg(p.slot_scale + slot) : 0.0f;
            s_row[tid] = placed ? r : -1;
            s_scale[tid] = scale;
            s_coef[tid] = placed ? __fmul_rn(__ldg(p.topk_weights + i), scale) : 0.0f;
        }
        for (int q = tid; q < nw * kMaxTopKDevice; q += blockDim.x) (&s_dot[0][0])[q] = 0.0f;
        __syncthreads();
        const uint4 *dy = p.dy + (size_t)t * p.hv;
        for (int base = 0; base < p.hv; base += blockDim.x * U) {
            uint4 g[U], v[U], nv[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int c = base + u * blockDim.x + tid;
                g[u] = c < p.hv ? ld_stream_v4(dy + c) : make_uint4(0u, 0u, 0u, 0u);
                const int r0 = s_row[0];
                v[u] = (c < p.hv && r0 >= 0) ? ld_stream_v4(p.buf + (size_t)r0 * p.hv + c) : make_uint4(0u, 0u, 0u, 0u);
            }
            for (int j = 0; j < k; ++j) {
                const int r = s_row[j], rn = j + 1 < k ? s_row[j + 1] : -1;
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    const int c = base + u * blockDim.x + tid;
                    nv[u] = (c < p.hv && rn >= 0) ? ld_stream_v4(p.buf + (size_t)rn * p.hv + c) : make_uint4(0u, 0u, 0u, 0u);
                }
                float dot = 0.0f;
                const float coef = s_coef[j];
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    const int c = base + u * blockDim.x + tid;
                    if (c >= p.hv || r < 0) continue;
                    const __nv_bfloat162 *a = reinterpret_cast<const __nv_bfloat162 *>(&v[u]);
                    const __nv_bfloat162 *b = reinterpret_cast<const __nv_bfloat162 *>(&g[u]);
                    float o[8];
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        const float2 fa = __bfloat1622float2(a[q]), fb = __bfloat1622float2(b[q]);
                        dot = __fmaf_rn(fa.x, fb.x, dot);
                        dot = __fmaf_rn(fa.y, fb.y, dot);
                        o[2 * q] = coef * fb.x; o[2 * q + 1] = coef * fb.y;
                    }
                    st_stream_v4(p.d_buf + (size_t)r * p.hv + c, pack_bf16x8(o));
                }
#pragma unroll
                for (int off = 16; off > 0; off >>= 1) dot += __shfl_xor_sync(0xffffffffu, dot, off);
                if (lane == 0) s_dot[warp][j] += dot;
#pragma unroll
                for (int u = 0; u < U; ++u) v[u] = nv[u];
            }
        }
        __syncthreads();
        if (tid < k) {
            float dot = 0.0f;
            for (int w = 0; w < nw; ++w) dot += s_dot[w][tid];
            p.d_weights[(size_t)t * k + tid] = s_row[tid] >= 0 ? s_scale[tid] * dot : 0.0f;
        }
    }
}

struct RouteBackwardParams {
    const float *logits;         // [T,E], read for sigmoid scores only
    const int32_t *topk_ids;     // [T,k]
    const float *topk_weights;   // [T,k]
    const float *d_weights;      // [T,k]
    float *d_logits;             // [T,E]
    int T, E, k;
    int sigmoid;
    float inv_scale;             // 1 / route_scale
};

constexpr int kRouteBwdThreads = 256;

// A warp per token: lanes j < k form the k gradients, the row of d_logits is cleared and the k values
// written into it (__syncwarp orders the two).  Lanes that name the same expert (possible only where
// routing ran out of experts and reported it) all write the sum of their values.
__global__ void __launch_bounds__(kRouteBwdThreads) k_route_backward(RouteBackwardParams p)
{
    const unsigned full = 0xffffffffu;
    const int lane = threadIdx.x & 31;
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const long long nwarps = (long long)gridDim.x * (kRouteBwdThreads / 32);
    for (long long t = (long long)blockIdx.x * (kRouteBwdThreads / 32) + (threadIdx.x >> 5); t < p.T; t += nwarps) {
        float w = 0.0f, g = 0.0f, slope = 1.0f;
        int id = -1;
        if (lane < p.k) {
            const size_t i = (size_t)t * p.k + lane;
            id = __ldg(p.topk_ids + i);
            w = __ldg(p.topk_weights + i);
            g = __ldg(p.d_weights + i);
            if ((unsigned)id >= (unsigned)p.E) id = -1;
            if (p.sigmoid && id >= 0) slope = sigmoid_spec(-__ldg(p.logits + (size_t)t * p.E + id));   // 1 - sigmoid(l) without cancellation
        }
        // g_j - sum_i p_i g_i as sum_i p_i (g_j - g_i) (the p_i = w_i / route_scale add up to 1): nothing
        // cancels where one expert has nearly all of the weight
        float diff = 0.0f;
        for (int i = 0; i < p.k; ++i) {
            const float wi = __shfl_sync(full, w, i), gi = __shfl_sync(full, g, i);
            diff += wi * p.inv_scale * (g - gi);
        }
        const float d = w * diff * slope;
        float sum = 0.0f;
        for (int j = 0; j < p.k; ++j) {
            const int oid = __shfl_sync(full, id, j);
            const float od = __shfl_sync(full, d, j);
            sum += oid == id ? od : 0.0f;
        }
        float *row = p.d_logits + (size_t)t * p.E;
        if ((p.E & 3) == 0) {
            for (int e = lane * 4; e < p.E; e += 128) *reinterpret_cast<float4 *>(row + e) = make_float4(0.f, 0.f, 0.f, 0.f);
        } else {
            for (int e = lane; e < p.E; e += 32) row[e] = 0.0f;
        }
        __syncwarp();
        if (id >= 0) row[id] = sum;
        __syncwarp();
    }
}

}  // namespace moe
