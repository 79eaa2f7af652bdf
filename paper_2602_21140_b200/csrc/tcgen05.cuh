// tcgen05, TMEM, TMA and cluster instructions that the product kernels share, and the host side of a tensor map (sm_100a).
#pragma once

#include <cuda.h>

#include <mutex>

#include "device_utils.cuh"

namespace moe {

// CG = CTAs that work on one MMA (1, or 2: a cluster of two SMs, each with half of the features in its
// TMEM and half of the row operand in its shared memory; the first CTA issues for both).

template <int CG>
__device__ __forceinline__ void tmem_alloc(uint32_t *slot, uint32_t cols)
{
    if (CG == 1) asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_addr(slot)), "r"(cols) : "memory");
    else asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_addr(slot)), "r"(cols) : "memory");
}

template <int CG>
__device__ __forceinline__ void tmem_dealloc(uint32_t base, uint32_t cols)
{
    if (CG == 1) {
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(base), "r"(cols));
    } else {
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;");
        asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(base), "r"(cols));
    }
}

// Arrive on `bar` (with CG = 2: on that barrier of both CTAs) when everything issued so far is done.
template <int CG>
__device__ __forceinline__ void mma_commit(uint64_t *bar)
{
    if (CG == 1)
        asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(smem_addr(bar)) : "memory");
    else
        asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(smem_addr(bar)),
                     "h"((uint16_t)3)
                     : "memory");
}

// 16 lanes x 32 columns in the fragment layout: v[4 i + 2 j + e] is lane 8 j + (thread / 4), column 8 i + 2 (thread % 4) + e
__device__ __forceinline__ void tmem_ld_fragment(uint32_t addr, uint32_t *r)
{
    asm volatile(
        "tcgen05.ld.sync.aligned.16x256b.x4.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]),
          "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
        : "r"(addr));
}

// 32 lanes: v[16 h + ...] for the lanes from 16 h on
__device__ __forceinline__ void tmem_ld_fragments(uint32_t addr, uint32_t (&r)[32])
{
#pragma unroll
    for (int h = 0; h < 2; ++h) tmem_ld_fragment(addr + ((uint32_t)(16 * h) << 16), r + 16 * h);
}

__device__ __forceinline__ void tmem_wait_ld() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tc_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_async_shared() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

__device__ __forceinline__ bool mbar_test_wait(uint64_t *bar, unsigned parity)
{
    unsigned ok;
    asm volatile("{\n\t.reg .pred p;\n\tmbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}"
                 : "=r"(ok) : "r"(smem_addr(bar)), "r"(parity) : "memory");
    return ok != 0;
}

__device__ __forceinline__ void mbar_arrive(uint64_t *bar)
{
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(smem_addr(bar)) : "memory");
}

__device__ __forceinline__ uint32_t cluster_rank()
{
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}

// The address of a barrier in the first CTA of the pair (its own for CG = 1).
template <int CG>
__device__ __forceinline__ uint32_t lead_addr(uint64_t *bar)
{
    if (CG == 1) return smem_addr(bar);
    uint32_t r;
    asm volatile("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(r) : "r"(smem_addr(bar)));
    return r;
}

// Arrival at the first CTA's barrier.  What it announces lies in this CTA's shared memory or TMEM, behind a proxy
// fence or a tcgen05 fence, and is read there by asynchronous units alone.  The PTX memory model orders it for the
// issuing thread of the other CTA only with a release of cluster scope, which also waits for this thread's loads and
// stores in global memory (1500 cycles a stage here).  So this relies on how the hardware does it: the fence has
// completed before the arrival leaves.  The tests compare pairs with single CTAs bit for bit.
template <int CG>
__device__ __forceinline__ void mbar_arrive_lead(uint64_t *bar)
{
    if (CG == 1) mbar_arrive(bar);
    else asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(lead_addr<2>(bar)) : "memory");
}

__device__ __forceinline__ void cluster_sync()
{
    asm volatile("barrier.cluster.arrive.aligned;" ::: "memory");
    asm volatile("barrier.cluster.wait.aligned;" ::: "memory");
}

// Tells the roles of a CTA, or of both CTAs of a pair, to leave.  (The other CTA is there: neither passes the last cluster_sync
// alone.)
template <int CG>
__device__ __forceinline__ void give_up(volatile int *quit)
{
    *quit = 1;
    if (CG == 2)
        asm volatile("{\n\t.reg .u32 a;\n\tmapa.shared::cluster.u32 a, %0, %1;\n\tst.shared::cluster.u32 [a], %2;\n\t}" ::"r"(
                         smem_addr(const_cast<int *>(quit))),
                     "r"(cluster_rank() ^ 1u), "r"(1)
                     : "memory");
}

// Tile loads into this CTA's shared memory; `bar` is a lead_addr.
template <int CG>
__device__ __forceinline__ void tma_2d(void *dst, const CUtensorMap *map, int x, int y, uint32_t bar)
{
    if (CG == 1)
        asm volatile("cp.async.bulk.tensor.2d.shared::cta.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];" ::"r"(
                         smem_addr(dst)),
                     "l"(map), "r"(x), "r"(y), "r"(bar)
                     : "memory");
    else
        asm volatile(
            "cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes.cta_group::2 [%0], [%1, {%2, %3}], [%4];" ::"r"(
                smem_addr(dst)),
            "l"(map), "r"(x), "r"(y), "r"(bar)
            : "memory");
}

template <int CG>
__device__ __forceinline__ void tma_3d(void *dst, const CUtensorMap *map, int x, int y, int z, uint32_t bar)
{
    if (CG == 1)
        asm volatile(
            "cp.async.bulk.tensor.3d.shared::cta.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(
                smem_addr(dst)),
            "l"(map), "r"(x), "r"(y), "r"(z), "r"(bar)
            : "memory");
    else
        asm volatile(
            "cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes.cta_group::2 [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(
                smem_addr(dst)),
            "l"(map), "r"(x), "r"(y), "r"(z), "r"(bar)
            : "memory");
}

// Weight rows as sixteens of {8 even, 8 odd} rows, of a map over {a row, eight rows of one parity, the parities, the sixteens,
// the slots}
template <int CG>
__device__ __forceinline__ void tma_pairs(void *dst, const CUtensorMap *map, int x, int sixteen, int slot, uint32_t bar)
{
    if (CG == 1)
        asm volatile(
            "cp.async.bulk.tensor.5d.shared::cta.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %5, %5, %3, %4}], [%6];" ::"r"(
                smem_addr(dst)),
            "l"(map), "r"(x), "r"(sixteen), "r"(slot), "r"(0), "r"(bar)
            : "memory");
    else
        asm volatile(
            "cp.async.bulk.tensor.5d.shared::cluster.global.tile.mbarrier::complete_tx::bytes.cta_group::2 [%0], [%1, {%2, %5, %5, %3, %4}], [%6];" ::"r"(
                smem_addr(dst)),
            "l"(map), "r"(x), "r"(sixteen), "r"(slot), "r"(0), "r"(bar)
            : "memory");
}

__device__ __forceinline__ bool elect_one()
{
    uint32_t r;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(r));
    return r != 0;
}

// ------------------------------------------------------------------------- host

typedef CUresult (*EncodeTiled)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *,
                                const cuuint32_t *, const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle,
                                CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

inline EncodeTiled encode_fn()
{
    static std::once_flag once;
    static EncodeTiled fn = nullptr;
    std::call_once(once, [] {
        void *f = nullptr;
        cudaDriverEntryPointQueryResult q;
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &f, 12000, cudaEnableDefault, &q) == cudaSuccess &&
            q == cudaDriverEntryPointSuccess)
            fn = reinterpret_cast<EncodeTiled>(f);
    });
    return fn;
}

inline bool encode(CUtensorMap *map, CUtensorMapDataType type, CUtensorMapSwizzle swizzle, const void *ptr, int rank, const cuuint64_t *dims,
            const cuuint64_t *strides, int box_cols, int box_rows, int box_2 = 1, int box_3 = 1)
{
    const cuuint32_t box[5] = {(cuuint32_t)box_cols, (cuuint32_t)box_rows, (cuuint32_t)box_2, (cuuint32_t)box_3, 1u}, one[5] = {1u, 1u, 1u, 1u, 1u};
    return encode_fn()(map, type, rank, const_cast<void *>(ptr), dims, strides, box, one, CU_TENSOR_MAP_INTERLEAVE_NONE,
                       swizzle, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

}  // namespace moe
