// K_mx_scatter: the scatter of a dispatch with 4-bit rows.  Every token's bf16 row is read once,
// quantised once in registers and its codes and scales written to its k rows of the
// expert-contiguous send buffer: 2H + k * 17H/32 bytes per token against (1 + k) * 2H of the bf16
// scatter (at H = 7168, k = 8: 44.8 KB against 129 KB).
//
// A warp works on 1024 columns of one token, with a grid of as many warps as there are such pieces: CTAs start as
// others finish, and SMs do not get equal shares of HBM (route and scatter of 8192 tokens of 7168, k = 8: 77 us;
// 91 us with the pieces dealt to the warps of a resident grid, 87-92 us with longer pieces).  Four coalesced 16-byte loads per lane, the block maxima by
// two shuffles within each quad of lanes, then a 4 x 4 transpose of the code words inside the quad so
// that every lane holds the whole 16 bytes of one block.  The transpose is done once and pays k
// times: a row piece leaves as one 16-byte store per lane instead of four 4-byte ones.
#pragma once

#include "mx_format.cuh"
#include "scatter_kernels.cuh"

namespace moe {

struct MxScatterParams {
    ScatterParams s;         // x, indices and outputs of the permutation; `send` is not used
    uint8_t *codes;          // [T*k, H/2]
    uint8_t *scales;         // [T*k, pitch]
    int pitch;
};

__global__ void __launch_bounds__(kScatterThreads) k_mx_scatter(MxScatterParams p)
{
    const unsigned full = 0xffffffffu;
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const int lane = lane_id();
    const int hv = p.s.hv;                                   // units of eight elements per row
    const int pieces = (hv + 127) / 128;                     // 1024-column pieces per row
    const long long it = (long long)blockIdx.x * (kScatterThreads / 32) + (threadIdx.x >> 5);
    if (it >= (long long)p.s.T * pieces) return;
    const int t = (int)(it / pieces), c = (int)(it % pieces);
    const size_t code_row = (size_t)hv * 4;                  // H/2 bytes
    const uint4 *src = p.s.x + (size_t)t * hv;
    uint4 in[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int u = c * 128 + 32 * i + lane;
        in[i] = u < hv ? ld_stream_v4(src + u) : make_uint4(0u, 0u, 0u, 0u);
    }
    // as in k_scatter_vec: x is an input of the dispatch, only the destinations wait
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int row = resolve_row(p.s, t, lane, c == 0);
    uint32_t w[4], s[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = mx_quantize8_bf16(in[i], s[i]);
    const uint32_t scale = mx_transpose(w, s, lane);
    const int block = c * 32 + mx_block_of_lane(lane);       // block of the row
    const bool inside = block * 4 < hv;
    const bool pad = !inside && block < p.pitch;             // padding of the row of scales: written as 0
    const uint4 out = make_uint4(w[0], w[1], w[2], w[3]);
    for (int j = 0; j < p.s.k; ++j) {
        const int r = __shfl_sync(full, row, j);
        if (r < 0) continue;
        if (inside) *reinterpret_cast<uint4 *>(p.codes + (size_t)r * code_row + (size_t)block * 16) = out;
        if (inside || pad) p.scales[(size_t)r * p.pitch + block] = inside ? (uint8_t)scale : (uint8_t)0;
    }
}

}  // namespace moe
