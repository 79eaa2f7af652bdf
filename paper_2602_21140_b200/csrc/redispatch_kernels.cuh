// K_redispatch: the send buffer of a dispatch once more, from its tokens' rows in 8 bits (mx8_format.cuh).
//
// A backward pass needs the experts' rows again (for the gradient of their first matrices), which are k copies of every token's
// row: kept as they are they take 2 H k bytes a token, kept as tokens in 8 bits 33/32 H.  A token's codes are read and
// turned into bf16 once, in registers, and stored k times, so the kernel is bound by its stores (2 H k bytes a token).
//
// A warp takes (token, piece of 32 * U units of eight elements), with as many warps in the grid as there are pieces.
#pragma once

#include "mx8_format.cuh"
#include "scatter_kernels.cuh"

namespace moe {

struct RedispatchParams {
    const uint2 *codes;      // [T, H]
    const uint8_t *scales;   // [T, pitch]
    const int32_t *dst_row;  // [T*k]
    uint4 *send;             // [T*k, H] bf16
    int T, k, hv, pitch;     // hv: units of a row
};

template <int U>
__global__ void __launch_bounds__(kScatterThreads) k_redispatch(RedispatchParams p)
{
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int lane = lane_id(), pieces = (p.hv + 32 * U - 1) / (32 * U);
    const long long it = (long long)blockIdx.x * (kScatterThreads / 32) + (threadIdx.x >> 5);
    if (it >= (long long)p.T * pieces) return;
    const int t = (int)(it / pieces), c0 = (int)(it % pieces) * (32 * U) + lane;
    int row = -1;
    if (lane < p.k) row = __ldg(p.dst_row + (size_t)t * p.k + lane);
    uint2 c[U];
    uint32_t s[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int at = c0 + 32 * u;
        if (at < p.hv) {
            c[u] = __ldg(p.codes + (size_t)t * p.hv + at);
            s[u] = __ldg(p.scales + (size_t)t * p.pitch + (at >> 2));
        }
    }
    uint4 v[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        if (c0 + 32 * u >= p.hv) continue;
        float f[8];
        mx8_unpack4(c[u].x, f); mx8_unpack4(c[u].y, f + 4);
        const float scale = mx_scale_value(s[u]);
        uint32_t w[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            // a code has four significant bits: exact in bf16 unless the scale leaves its range
            const __nv_bfloat162 h = __floats2bfloat162_rn(f[2 * q] * scale, f[2 * q + 1] * scale);
            w[q] = *reinterpret_cast<const uint32_t *>(&h);
        }
        v[u] = make_uint4(w[0], w[1], w[2], w[3]);
    }
    const long long rows = (long long)p.T * p.k;
    for (int j = 0; j < p.k; ++j) {
        const int r = __shfl_sync(0xffffffffu, row, j);
        if (r < 0 || r >= rows) continue;                    // an assignment that was not placed
        uint4 *dst = p.send + (size_t)r * p.hv;
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (c0 + 32 * u < p.hv) st_stream_v4(dst + c0 + 32 * u, v[u]);
    }
}

}  // namespace moe
