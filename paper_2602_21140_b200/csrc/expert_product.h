// Launch interface of the experts' products in 16 bits (expert_product.cu), used by the host side in moe_route.cu.
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

#include "device_utils.cuh"
#include "mx_product.h"

namespace moe {

enum class ExpertOp {
    kProduct,        // y[r, n] = sum_k a[r, k] w[p, n, k]
    kGated,          // h = SwiGLU of the same over pairs of rows of w, and z, the sums, if asked for
    kTransposed,     // y[r, n] = sum_k a[r, k] w[p, k, n]
    kGatedBackward,  // the same sum is dh; dz and h from it and z
    kWeightGrad,     // y[p, m, n] = sum_r a[r, m] b[r, n] over the slot's segment
};

struct ExpertArgs {
    ExpertOp op;
    const void *a;                       // [rows, K] bf16 (kWeightGrad: [rows, M])
    const void *b;                       // kWeightGrad: [rows, N] bf16
    long long rows;
    const int32_t *slot_counts;          // [P] device
    const int32_t *slot_offsets;         // [P] device
    int P;
    const void *w;                       // [P, N, K] bf16, transposed: [P, K, N]
    int N, K, M;                         // N: columns of the sums (kGated: 2 * hidden features)
    void *y;                             // [rows, N] bf16; kGated, kGatedBackward: h [rows, features]; kWeightGrad: [P, M, N]
    void *z;                             // kGated: out, NULL or [rows, N]; kGatedBackward: in, [rows, 2 N]; bf16 or 8-bit codes
    uint8_t *z_scales;                   // NULL: z is bf16
    void *dz;                            // kGatedBackward: out, [rows, 2 N] bf16
    bool f32, add;                       // kWeightGrad: y is fp32 and not bf16; the sums are added to it (fp32 only)
    Control *ctl;
    unsigned spin_limit;
    int sm_count;
    int device;                          // the current one
    bool pdl;
};

// Whether sizes fit the kernels' numbers (see product_fits): features, rows and tiles are counted in int.
inline bool expert_product_fits(long long rows, long long n, long long k, int P)
{
    if (rows > kMaxRows || n > kMaxFeatures || k > kMaxFeatures) return false;
    return (n + 127) / 128 * (P + rows / 32) < kTooManyTiles && n * k * 2 < (1ll << 39);
}
inline bool weight_grad_fits(long long rows, long long m, long long n, int P)
{
    if (rows > kMaxRows || m > kMaxFeatures || n > kMaxFeatures) return false;
    return (m + 255) / 256 * ((n + 255) / 256) < kTooManyTiles / P && m * n * 4 < (1ll << 39);
}

// Polls allowed to a wait that lasts through several tiles: `so_far`, and for one more of `steps` stages what a role that works on it
// is allowed for the tile and its stages (512 clocks a stage; a poll takes 39 clocks at least, and 7800 where the hardware waits
// for the barrier as long as it does).  Bounded, by a minute of the longer polls, and without overflow.
constexpr unsigned kMostPatience = 1u << 24;
__host__ __device__ inline unsigned more_patience(unsigned so_far, unsigned spin_limit, int steps)
{
    const unsigned tile = (spin_limit < kMostPatience ? spin_limit : kMostPatience) + 64u * (unsigned)steps, sum = so_far + tile;
    return sum < kMostPatience ? sum : kMostPatience;
}

cudaError_t expert_product_launch(const ExpertArgs &a, cudaStream_t st);

}  // namespace moe
