// Launch interface of the experts' products (mx_product.cu), used by the host side in moe_route.cu.
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

#include "device_utils.cuh"

namespace moe {

// Sums of tile counts stop at kTooManyTiles.  Segments that do not overlap stay below it (the host checks that); counts
// left behind by a dispatch that gave up may not.  Two sums that have both stopped there still add up to an int.
constexpr int kTooManyTiles = 1 << 29;
__host__ __device__ inline int tiles_sum(int a, int b) { return min(a + b, kTooManyTiles); }

// Whether the sizes of a product fit the kernels' numbers: features are counted in int, rounded up to the two tiles
// of a pair; rows are coordinates of a tensor map; tile numbers stay below kTooManyTiles; strides below 2^40 bytes.
constexpr int kMaxFeatures = 1 << 30, kMaxRows = 1 << 30;
inline bool product_fits(long long rows, long long n_out, long long n_in, int P)
{
    if (rows > kMaxRows || n_out > kMaxFeatures) return false;
    return (n_out + 127) / 128 * (P + rows / 32) < kTooManyTiles && n_out * (n_in / 2) < (1ll << 40);
}

struct MxProductArgs {
    const uint8_t *a_codes, *a_scales;   // [rows, K/2], [rows, pitch(K)]
    long long rows;
    const int32_t *slot_counts;          // [P] device
    const int32_t *slot_offsets;         // [P] device
    int P;
    const uint8_t *w_codes, *w_scales;   // [P, N, K/2], [P, N, pitch(K)]
    int N, K;
    bool gated;                          // SwiGLU over row pairs, 4-bit output of N/2 columns
    void *y;                             // plain: [rows, N] bf16
    uint8_t *h_codes, *h_scales;         // gated: [rows, N/4], [rows, pitch(N/2)]
    Control *ctl;
    unsigned spin_limit;
    int sm_count;
    int device;                          // the current one
    bool pdl;
};

cudaError_t mx_product_launch(const MxProductArgs &a, cudaStream_t st);

}  // namespace moe
