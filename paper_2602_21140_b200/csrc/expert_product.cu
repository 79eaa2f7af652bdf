// The experts' products on bf16 rows and their gradients, on tcgen05.mma kind::f16 (fp32 accumulation).  For every physical
// slot p and the rows r of its segment:
//     kProduct         y[r, n] = sum_k a[r, k] w[p, n, k]
//     kGated           the same sums z over the pairs of rows 2i, 2i + 1 of w, and h[r, i] = silu(z[2i]) z[2i + 1]
//     kTransposed      y[r, n] = sum_k a[r, k] w[p, k, n]                       (gradient by the rows)
//     kGatedBackward   the same sums dh, and with g = z[2i], u = z[2i + 1], s = 1 / (1 + exp(-g)):
//                      dz[2i] = dh u s (1 + g (1 - s)), dz[2i + 1] = dh g s, h = g s u
//     kWeightGrad      y[p, m, n] = sum_r a[r, m] b[r, n]                       (gradient by the weights)
//
// Weights are the M operand and rows the N operand of the first four, so a segment costs its own length rounded up to 32,
// from one token to hundreds, and a tile's accumulator is [128 lanes = features] x [columns = rows] in TMEM.  The weight
// gradient has the features of a as M, those of b as N, and rows as K.  K goes in stages of 64: a K-major operand (w, a of
// the products) has 128 bytes of a row, one 128-byte swizzle span; an operand that runs along M or N in memory (w of the
// transposed products, both of the weight gradient) has 64 lines of 64 features, with the same swizzle.
//
// A pair of persistent CTAs per two SMs works on one MMA (cta_group::2): each has 128 of a tile's 256 features in its TMEM and
// shared memory, and half of its rows.  In each CTA
//   warps 0-7   epilogue, two groups of four (a warp reads one quarter of the TMEM lanes): TMEM -> registers ->
//               shared memory -> HBM, 32 columns at a time, the groups taking turns
//   warp 8      TMA loads
//   warp 9      the MMAs, from one thread
// The accumulator is double buffered, so the epilogue of a tile runs under the products of the next.
//
// What bounds it: with many rows the tensor cores, under the power cap (at 32 slots of 1024 rows, 4096 x 1024, they are busy for
// 90 % of the gated product and 92 % of the gradient by the rows, at 1.39 GHz).  A stage of 64 is 32 KB a CTA in the 512 clocks of its
// MMAs, all that an SM gets from L2, so nothing else may use that path: prefetching stages into L2 by TMA cost 15 %.  The
// gradient of the gate (77 %) and the weights' (85 %, in fp32 66 %) move as many bytes of HBM as products, and wait for loads.
// With few rows HBM: one row for 8 slots of 7168 x 2048 takes 77 + 46 us, whose weights take 72 + 36.  Single CTAs with tiles of
// 64 rows were as fast up to 64 rows a slot and took up to 2.4 times as long with 200.
#include "expert_product.h"

#include <algorithm>
#include <mutex>
#include <type_traits>

#include "mx8_format.cuh"
#include "tcgen05.cuh"

namespace {

using namespace moe;

constexpr int CG = 2;                      // CTAs of a pair, which work on one MMA
constexpr int NT = 256;                    // rows (N) of a tile at most
constexpr int kFeat = 128;                 // features (M) per CTA and tile
constexpr int kStageK = 64;                // elements of K per stage
constexpr int kLine = 128;                 // bytes of a line of an operand tile: 64 elements
constexpr int kChunk = 64 * kLine;         // 64 features x 64 K of an operand that runs along its features
constexpr int kATile = kFeat * kLine;      // 16 KB
constexpr int kEpiWarps = 8, kTmaWarp = kEpiWarps, kMmaWarp = kEpiWarps + 1;
constexpr int kMaxStages = 10;
constexpr int kBand = 8;                   // tiles of rows (or of n) that are worked on side by side, see tile_at

// ------------------------------------------------------------------ tcgen05 in PTX (the rest: tcgen05.cuh)

__device__ __forceinline__ void mma_bf16(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, bool accumulate)
{
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
                 "tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"((uint32_t)accumulate)
                 : "memory");
}

// 32 lanes x 32 columns: v[c] is column c of lane threadIdx.x % 32
__device__ __forceinline__ void tmem_ld_lanes(uint32_t addr, uint32_t (&r)[32])
{
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, %18, "
        "%19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]),
          "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]),
          "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]),
          "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
        : "r"(addr));
}

// 32 lanes x 16 columns
__device__ __forceinline__ void tmem_ld_lanes(uint32_t addr, uint32_t (&r)[16])
{
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]),
          "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
        : "r"(addr));
}

// Shared-memory matrix descriptors: start and strides in 16-byte units, version 1 (sm_100), 128-byte swizzle.
// Along K: eight rows of 128 bytes are an atom, atoms 1024 bytes apart.  Along M or N: eight lines (K) of 64 elements
// are an atom, the next eight of K 1024 bytes on, the next 64 elements a chunk on.
template <bool ALONG_K>
__device__ __forceinline__ uint64_t desc_tile(uint32_t addr)
{
    const uint64_t lead = ALONG_K ? 1 : kChunk >> 4;
    return (uint64_t)((addr >> 4) & 0x3fffu) | (lead << 16) | (64ull << 32) | (1ull << 46) | (2ull << 61);
}
// bytes from one K = 16 of a tile to the next, in the descriptor's units
template <bool ALONG_K>
constexpr uint32_t kDescStep = (ALONG_K ? 16 * 2 : 16 * kLine) >> 4;

// Instruction descriptor of kind::f16: fp32 accumulators (1 at bit 4), A and B bf16 (1 at 7 and 10), operands that run
// along M or N (15 and 16), N / 8 at bit 17, M / 16 at bit 24.
template <bool A_ALONG_K, bool B_ALONG_K>
__device__ __forceinline__ uint32_t idesc_bf16(int n)
{
    return (1u << 4) | (1u << 7) | (1u << 10) | (A_ALONG_K ? 0u : 1u << 15) | (B_ALONG_K ? 0u : 1u << 16) | ((uint32_t)(n >> 3) << 17) |
           ((uint32_t)(CG * kFeat >> 4) << 24);
}

// ------------------------------------------------------------------------ tiles

struct KernelParams {
    const int32_t *slot_counts, *slot_offsets;
    long long rows;
    int P, N, K, M;
    int ring;                      // bytes
    void *y;                       // kGated, kGatedBackward: h
    void *z;
    uint8_t *z_scales;
    __nv_bfloat16 *dz;
    int add;
    Control *ctl;
    unsigned spin_limit;
};

// feat: first feature (M) of the tile; row, rows: first row and rows, of the tile (products) or of its whole segment (weight
// gradient); col: first column of a weight gradient's tile
struct Tile {
    int slot, feat, row, rows, col;
};

// Rows of slot p that can be worked on: counts and offsets come from device memory, so a segment
// that leaves the row buffer is cut (or dropped) instead of followed.
__device__ __forceinline__ int segment(const KernelParams &p, int s, int &first)
{
    first = __ldg(p.slot_offsets + s);
    const long long c = __ldg(p.slot_counts + s);
    if (first < 0 || c <= 0 || first >= p.rows) return 0;
    return (int)min(c, p.rows - first);
}

// A segment of c rows is cut into the fewest tiles of at most NT rows, of equal size (to whole pieces of the
// epilogue, 32 rows: only a segment's last tile leaves part of one).
__device__ __forceinline__ int row_tiles(int c) { return (c + NT - 1) / NT; }

// Neighbours in the order of the tiles run at the same time and share what they read through L2.  So the nt tiles of
// rows of a slot are dealt in bands of kBand, and in a band all feature tiles one after the other, rows innermost: 74
// pairs work on 8 tiles of rows by 9 of features, and a band's rows stay in L2 while the weights go by.  (All rows of a
// segment innermost would read the rows from HBM again for every tile of features, once they outgrow L2.)
__device__ __forceinline__ void in_bands(int local, int feats, int nt, int &f, int &r)
{
    const int band = local / (feats * kBand), wide = min(kBand, nt - band * kBand);
    local -= band * feats * kBand;
    f = local / wide;
    r = band * kBand + local - f * wide;
}

template <ExpertOp OP>
__device__ __forceinline__ Tile tile_at(const KernelParams &p, const int *ends, int index)
{
    Tile t;
    int f, r;
    if (OP == ExpertOp::kWeightGrad) {
        const int mt = (p.M + CG * kFeat - 1) / (CG * kFeat), nt = (p.N + NT - 1) / NT;
        t.slot = index / (mt * nt);
        in_bands(index - t.slot * mt * nt, mt, nt, f, r);
        t.rows = segment(p, t.slot, t.row);
        t.feat = f * (CG * kFeat); t.col = r * NT;
        return t;
    }
    int lo = 0, hi = p.P - 1;                        // first slot whose inclusive end is beyond the index
#pragma unroll 1
    while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if (ends[mid] > index) hi = mid; else lo = mid + 1;
    }
    int first;
    const int c = segment(p, lo, first), nt = row_tiles(c), size = ((c + nt - 1) / nt + 31) & ~31;
    in_bands(index - (lo ? ends[lo - 1] : 0), (p.N + CG * kFeat - 1) / (CG * kFeat), nt, f, r);
    t.slot = lo; t.feat = f * (CG * kFeat); t.col = 0;
    t.row = first + r * size;
    t.rows = min(size, c - r * size);                // may be <= 0 for the last tile of an uneven cut
    return t;
}

// N of a tile's MMAs: its rows (weight gradient: columns) rounded up to what the instruction takes
template <ExpertOp OP>
__device__ __forceinline__ int tile_n(const KernelParams &p, const Tile &t)
{
    const int n = OP == ExpertOp::kWeightGrad ? min(NT, p.N - t.col) : t.rows;
    return (n + 16 * CG - 1) & -(16 * CG);
}

// The tiles of a CTA (or pair of CTAs) of a grid of `step`, first, first + step, ..., as a warp sees them.  Finding a
// tile is a chain of dependent reads, so the lanes find the next 32 of them side by side and hand them out one by one.
// The fields and the verdict are in uniform registers (a warp reduction writes those): what tcgen05 and TMA
// instructions take comes from uniform registers.
template <ExpertOp OP>
struct TileStream {
    const KernelParams &p;
    const int *ends;
    const int tiles;
    int base, at;
    Tile mine;
    __device__ TileStream(const KernelParams &p_, const int *ends_, int tiles_)
        : p(p_), ends(ends_), tiles(tiles_), base(blockIdx.x / CG), at(32), mine{}
    {
    }
    __device__ bool next(Tile &t)                    // false when there are no more
    {
        while (true) {
            if (at == 32) {
                if (base >= tiles) return false;
                const int step = (int)gridDim.x / CG, i = base + (int)(threadIdx.x & 31) * step;
                mine.rows = 0; mine.slot = -1;
                if (i < tiles) mine = tile_at<OP>(p, ends, i);
                base += 32 * step;
                at = 0;
                __syncwarp();
            }
            const int slot = __shfl_sync(0xffffffffu, mine.slot, at);
            t.feat = (int)__reduce_max_sync(0xffffffffu, (unsigned)__shfl_sync(0xffffffffu, mine.feat, at));
            t.row = (int)__reduce_max_sync(0xffffffffu, (unsigned)__shfl_sync(0xffffffffu, mine.row, at));
            t.col = (int)__reduce_max_sync(0xffffffffu, (unsigned)__shfl_sync(0xffffffffu, mine.col, at));
            t.rows = __reduce_max_sync(0xffffffffu, __shfl_sync(0xffffffffu, mine.rows, at));
            ++at;
            if (!__any_sync(0xffffffffu, slot >= 0)) return false;
            t.slot = (int)__reduce_max_sync(0xffffffffu, (unsigned)slot);
            // a slot without rows has no tiles of products, and a gradient of zeros
            if (OP == ExpertOp::kWeightGrad || t.rows > 0) return true;
        }
    }
};

// Threads of a CTA.  Where the epilogue keeps sums in registers (FINE: 128 of a thread), the two issuing warps are
// filled up to a warpgroup, which hands registers to the two of the epilogue: 72 + 2 * 216 = 3 * 168, what the launch gives.
template <bool FINE> constexpr int kThreadsOf = FINE ? 384 : 32 * (kEpiWarps + 2);

template <ExpertOp OP, bool FINE>
struct Layout {
    static constexpr int kThreads = kThreadsOf<FINE>;
    static constexpr bool kGrad = OP == ExpertOp::kWeightGrad;
    static constexpr bool kAAlongK = OP == ExpertOp::kProduct || OP == ExpertOp::kGated;   // see desc_tile
    static constexpr bool kBAlongK = !kGrad;
    static constexpr bool kFragments = OP == ExpertOp::kGated;   // how the epilogue reads an accumulator
    static constexpr int kN = NT / CG;                        // rows (or columns) of a tile in this CTA
    static constexpr int kStage = kATile + kN * kLine;        // multiples of 1024: swizzle alignment
    static constexpr int kEpiWarp = 32 * kLine;               // a plane of 32 x 32 fp32 or 32 x 64 bf16
    static constexpr int kBars = 4 * kMaxStages + 5;
    static constexpr int kEpiOff = 0, kBarOff = kEpiWarps * kEpiWarp;
    static constexpr int kEndsOff = kBarOff + ((kBars * 8 + 16 + 8 * (kThreads / 32) + 15) & ~15);
    static constexpr int kSmem = 227 * 1024;
    static size_t fixed(int P) { return (kEndsOff + (kGrad ? 0 : (size_t)P * 4) + 1023) / 1024 * 1024; }
    static int ring(int P) { return (int)(kSmem - 1024 - fixed(P)) / kStage * kStage; }   // its bytes: whole stages at their largest
    static size_t bytes(int P) { return 1024 + fixed(P) + (size_t)ring(P); }
};

// Whether the last of `left` rows of a weight gradient's segment end inside a K = 16 of this stage.
__device__ __forceinline__ bool has_tail(int left) { return left < kStageK && (left & 15) != 0; }

// Both operands of a stage of a weight gradient, 64 features by 64 rows at a time; PEER: `bar` is in the first CTA.
template <bool PEER>
__device__ __forceinline__ void load_grad(unsigned char *a, unsigned char *b, const CUtensorMap *map_a, const CUtensorMap *map_b, int feat, int col,
                                          int row, uint32_t bar)
{
#pragma unroll
    for (int q = 0; q < kFeat / 64; ++q) tma_2d<PEER ? CG : 1>(a + q * kChunk, map_a, feat + q * 64, row, bar);
#pragma unroll
    for (int q = 0; q < NT / CG / 64; ++q) tma_2d<PEER ? CG : 1>(b + q * kChunk, map_b, col + q * 64, row, bar);
}

// The lines of a stage behind a segment, up to a whole K = 16, are made zero in both operands: they hold the next segment's rows
// (and a NaN there times a zero would still be one).  A line is 128 bytes of one k in each of the stage's chunks.  In the CTA whose
// thread issues the MMAs by that thread's warp:
__device__ __forceinline__ void clear_tail(unsigned char *stage, int bytes, int left, int lane)
{
    unsigned char *lines = stage + (lane & 7) * 16;
    for (int i = left; i < ((left + 15) & ~15); ++i)
        for (int q = (lane >> 3) * kChunk; q < bytes; q += 4 * kChunk) *reinterpret_cast<uint4 *>(lines + q + i * kLine) = make_uint4(0u, 0u, 0u, 0u);
    fence_async_shared();
    __syncwarp();
}

// In the other one by loads of zeros, of lines beyond the rows, which count their bytes at `bar` of the first CTA.  (Stores and an
// arrival there would need a release of cluster scope, 1500 clocks of it: the CTAs' shared memory is read by the first one's MMAs,
// and what orders a load's bytes for them is the barrier that every stage has.  128 x 511 rows, 2048 x 4096: 931 us; with an arrival
// that nothing orders 904, with the release 1488 for 1054 in an earlier state.)
struct ZeroMaps {
    CUtensorMap lines[4];                                      // boxes of 1, 2, 4 and 8 lines
};
constexpr int kTailChunks = (kFeat + NT / CG) / 64;            // of a stage
__device__ __forceinline__ int tail_lines(int left) { return 16 - (left & 15); }
__device__ __forceinline__ void load_zero_tail(unsigned char *stage, int left, const ZeroMaps &zeros, int beyond, uint32_t bar)
{
    int at = left;
#pragma unroll
    for (int b = 0; b < 4; ++b)
        if (tail_lines(left) & (1 << b)) {
#pragma unroll
            for (int q = 0; q < kTailChunks; ++q) tma_2d<CG>(stage + q * kChunk + at * kLine, &zeros.lines[b], 0, beyond, bar);
            at += 1 << b;
        }
}

// Bounded wait.  `quit` is shared by the CTA: the first role that gives up sets it in both, the others follow.
__device__ __forceinline__ bool wait_for(uint64_t *bar, unsigned parity, volatile int *quit, unsigned limit)
{
    unsigned spins = 0;
    while (!mbar_try_wait(bar, parity)) {
        if (++spins > limit || ((spins & 63u) == 0 && *quit)) { give_up<CG>(quit); return false; }
    }
    return true;
}

// ---------------------------------------------------------------------- epilogue

// s = 1 / (1 + exp(-g)), by the hardware's exp and reciprocal (2 and 1 units in the last place; the rounded argument of
// exp costs up to |g| 2^-24 relative besides: far below the bf16 that its results are rounded to).  Both flush to zero: below
// g = -87.3, where s is less than 2^-126, it is 0.  (The formula in 32 bits does the same from g = -88.7 on.)
__device__ __forceinline__ float sigmoid(float g)
{
    float e, r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(g * -1.44269504f));
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(1.0f + e));
    return r;
}

__device__ __forceinline__ uint32_t pack_bf16(float a, float b)
{
    const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t *>(&h);
}

// A warp's 32 features x 32 rows, turned round in shared memory: lane l of the accumulator is a feature, and afterwards
// lane l holds eight neighbouring features of row 8 i + l / 4, so that four lanes have 32 features of a row in a run.
// The 16-byte units of a row are permuted by the row, so that neither the stores (32 lanes of one row) nor the loads of 16
// bytes (two rows, every other unit) meet in a bank.
__device__ __forceinline__ void write_plane(float *plane, const uint32_t (&v)[32], int lane)
{
#pragma unroll
    for (int r = 0; r < 32; ++r) plane[r * 32 + (lane ^ ((r & 7) << 2))] = __uint_as_float(v[r]);
    __syncwarp();
}

__device__ __forceinline__ void read_eight(const float *plane, int i, int lane, float (&x)[8])
{
    const float4 *row = reinterpret_cast<const float4 *>(plane + (8 * i + (lane >> 2)) * 32);
    const int unit = ((lane & 3) * 2) ^ (lane >> 2);           // row % 8 = lane / 4
    const float4 a = row[unit], b = row[unit ^ 1];
    x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w; x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
}

// f: first of the warp's features, left: rows of the segment from the piece's first one, `row`, on.  The fp32 sums
// are rounded once.
__device__ __forceinline__ void store_rows(const KernelParams &p, const float *plane, int f, long long row, int left, int lane)
{
    f += (lane & 3) * 8;
    if (f >= p.N) return;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int r = 8 * i + (lane >> 2);
        float x[8];
        read_eight(plane, i, lane, x);
        if (r < left)
            *reinterpret_cast<uint4 *>(static_cast<__nv_bfloat16 *>(p.y) + (row + r) * p.N + f) =
                make_uint4(pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]), pack_bf16(x[4], x[5]), pack_bf16(x[6], x[7]));
    }
}

// 8 pairs x 32 rows of 16-bit values in the fragment layout, m[i] being rows 8 i + 2 (lane % 4) and the next: written
// as rows, `addr` being that of this lane's row.
__device__ __forceinline__ void store_transposed(uint32_t addr, const uint32_t (&m)[4])
{
    asm volatile("stmatrix.sync.aligned.m8n8.x4.trans.shared.b16 [%0], {%1, %2, %3, %4};" ::"r"(addr), "r"(m[0]), "r"(m[1]), "r"(m[2]), "r"(m[3])
                 : "memory");
}

// Rows of 16 pairs, 2 bytes each, in shared memory: where the eight of half c lie.
__device__ __forceinline__ int pairs_at(int r, int c) { return r * 32 + ((c ^ ((r >> 2) & 1)) << 4); }

// SwiGLU of 16 pairs x 32 rows, and the sums themselves where they are kept, in bf16 or in 8 bits (the warp's 32 sums of a
// row are one block).  The features of a gated product lie in TMEM as sixteens of 8 gates and their 8 up-projections, so that a thread has
// both of a pair: v[16 h + 4 i + e] and v[16 h + 4 i + 2 + e] for pair 8 h + lane / 4 and row 8 i + 2 (lane % 4) + e.  Two rows of a pair of
// codes or of outputs are a register, which stmatrix turns round.  (Through a plane of fp32, as in store_rows, the epilogue bounds short K: 32
// slots of 2048 rows, 1024 x 1024, 200 us and 246 with 8-bit sums instead of 169 and 222.  Rows without a gate have less to gain and
// were 2 % slower by fragments.)
__device__ __forceinline__ void store_gated(const KernelParams &p, const uint32_t (&v)[32], unsigned char *box, int f, long long row, int left,
                                            int lane)
{
    const uint32_t base = smem_addr(box);
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        uint32_t m[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float o[2];
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const float g = __uint_as_float(v[16 * h + 4 * i + e]);
                o[e] = g * sigmoid(g) * __uint_as_float(v[16 * h + 4 * i + 2 + e]);
            }
            m[i] = pack_bf16(o[0], o[1]);
        }
        store_transposed(base + pairs_at(lane, h), m);
    }
    unsigned char *codes = box + 1024, *gates = box + 1024, *ups = box + 2048;
    if (p.z_scales) {
        uint32_t most[4];                                      // of two rows each, in 16 bits
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            uint32_t a[2];
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                a[e] = 0;
#pragma unroll
                for (int q = 0; q < 4; ++q) a[e] = max(a[e], v[16 * (q >> 1) + 4 * i + 2 * (q & 1) + e] & 0x7fffffffu);
                // Rounded up to a bf16, two to a register: all that the scale asks is whether the mantissa is above 1.75, which
                // is one.  (Not up to infinity: the largest bf16 has the scale of all that lies between.)
                a[e] = a[e] >= 0x7f800000u ? a[e] >> 16 : min((a[e] + 0xffffu) >> 16, 0x7f7fu);
            }
            most[i] = a[0] | a[1] << 16;
#pragma unroll
            for (int off = 4; off < 32; off <<= 1) {
                const uint32_t o = __shfl_xor_sync(0xffffffffu, most[i], off);
                asm("max.u16x2 %0, %0, %1;" : "+r"(most[i]) : "r"(o));
            }
        }
        float inv[4][2];
        uint32_t keep[4];                                      // a block with a NaN or infinity has codes of 0
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t s0 = mx8_scale_byte(most[i] << 16), s1 = mx8_scale_byte(most[i] & 0xffff0000u);
            inv[i][0] = mx_inverse_scale(s0); inv[i][1] = mx_inverse_scale(s1);
            keep[i] = (s0 == 255u ? 0u : 0xffffu) | (s1 == 255u ? 0u : 0xffff0000u);
        }
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            uint32_t m[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t *w = &v[16 * h + 4 * i];
                m[i] = mx8_pack4(__uint_as_float(w[0]) * inv[i][0], __uint_as_float(w[2]) * inv[i][0], __uint_as_float(w[1]) * inv[i][1],
                                 __uint_as_float(w[3]) * inv[i][1]) & keep[i];
            }
            store_transposed(smem_addr(codes) + pairs_at(lane, h), m);
        }
        const int r = 8 * (lane >> 3) + 2 * (lane & 3) + ((lane >> 2) & 1);   // every row's scale by one lane
        const uint32_t two = lane < 16 ? (lane < 8 ? most[0] : most[1]) : (lane < 24 ? most[2] : most[3]);
        if (r < left && f < p.N)
            p.z_scales[(row + r) * mx_scale_pitch(p.N) + f / kMxBlock] = (uint8_t)mx8_scale_byte(lane & 4 ? two & 0xffff0000u : two << 16);
    } else if (p.z) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            uint32_t g[4], u[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t *w = &v[16 * h + 4 * i];
                g[i] = pack_bf16(__uint_as_float(w[0]), __uint_as_float(w[1]));
                u[i] = pack_bf16(__uint_as_float(w[2]), __uint_as_float(w[3]));
            }
            store_transposed(smem_addr(gates) + pairs_at(lane, h), g);
            store_transposed(smem_addr(ups) + pairs_at(lane, h), u);
        }
    }
    __syncwarp();
    const int c = lane & 1;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int r = 16 * i + (lane >> 1);
        if (r >= left || f >= p.N) continue;                   // N is a multiple of 32: all of the block or nothing
        *reinterpret_cast<uint4 *>(static_cast<__nv_bfloat16 *>(p.y) + (row + r) * (p.N / 2) + f / 2 + 8 * c) =
            *reinterpret_cast<const uint4 *>(box + pairs_at(r, c));
        if (p.z_scales) {
            *reinterpret_cast<uint4 *>(static_cast<uint8_t *>(p.z) + (row + r) * p.N + f + 16 * c) =
                *reinterpret_cast<const uint4 *>(codes + pairs_at(r, c));
        } else if (p.z) {
            const uint4 g = *reinterpret_cast<const uint4 *>(gates + pairs_at(r, c)), u = *reinterpret_cast<const uint4 *>(ups + pairs_at(r, c));
            uint4 *dst = reinterpret_cast<uint4 *>(static_cast<__nv_bfloat16 *>(p.z) + (row + r) * p.N + f + 16 * c);
            dst[0] = make_uint4(__byte_perm(g.x, u.x, 0x5410), __byte_perm(g.x, u.x, 0x7632), __byte_perm(g.y, u.y, 0x5410), __byte_perm(g.y, u.y, 0x7632));
            dst[1] = make_uint4(__byte_perm(g.z, u.z, 0x5410), __byte_perm(g.z, u.z, 0x7632), __byte_perm(g.w, u.w, 0x5410), __byte_perm(g.w, u.w, 0x7632));
        }
    }
}

// The kept sums of eight features (16 of them) of a row, asked for before the product of the piece is there.
struct Kept {
    uint4 v[2];
    uint32_t s;
};

__device__ __forceinline__ void load_kept(const KernelParams &p, int f, long long row, int left, int lane, Kept (&k)[4])
{
    const int at = 2 * (f + (lane & 3) * 8), cols = 2 * p.N;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int r = 8 * i + (lane >> 2);
        k[i].v[0] = k[i].v[1] = make_uint4(0u, 0u, 0u, 0u);
        k[i].s = 0u;
        if (r >= left || at >= cols) continue;
        if (p.z_scales) {
            k[i].v[0] = __ldg(reinterpret_cast<const uint4 *>(static_cast<const uint8_t *>(p.z) + (row + r) * cols + at));
            k[i].s = __ldg(p.z_scales + (row + r) * mx_scale_pitch(cols) + at / kMxBlock);
        } else {
            const uint4 *src = reinterpret_cast<const uint4 *>(static_cast<const __nv_bfloat16 *>(p.z) + (row + r) * cols + at);
            k[i].v[0] = __ldg(src);
            k[i].v[1] = __ldg(src + 1);
        }
    }
}

// Gradient of SwiGLU for 32 features x 32 rows, and its output once more for the gradient of the down matrix.
__device__ __forceinline__ void store_gated_backward(const KernelParams &p, const float *plane, int f, long long row, int left, int lane,
                                                     const Kept (&k)[4])
{
    f += (lane & 3) * 8;
    if (f >= p.N) return;                                      // N is a multiple of 16
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int r = 8 * i + (lane >> 2);
        float dh[8], z[16], h[8];
        read_eight(plane, i, lane, dh);
        if (p.z_scales) {
            const float scale = mx_scale_value(k[i].s);
            const uint32_t c[4] = {k[i].v[0].x, k[i].v[0].y, k[i].v[0].z, k[i].v[0].w};
#pragma unroll
            for (int q = 0; q < 4; ++q) mx8_unpack4(c[q], z + 4 * q);
#pragma unroll
            for (int q = 0; q < 16; ++q) z[q] *= scale;
        } else {
            const uint32_t c[8] = {k[i].v[0].x, k[i].v[0].y, k[i].v[0].z, k[i].v[0].w, k[i].v[1].x, k[i].v[1].y, k[i].v[1].z, k[i].v[1].w};
#pragma unroll
            for (int q = 0; q < 8; ++q) { z[2 * q] = __uint_as_float(c[q] << 16); z[2 * q + 1] = __uint_as_float(c[q] & 0xffff0000u); }
        }
        uint32_t d[8];
#pragma unroll
        for (int q = 0; q < 8; ++q) {
            const float g = z[2 * q], u = z[2 * q + 1], s = sigmoid(g), a = g * s;
            h[q] = a * u;
            d[q] = pack_bf16(dh[q] * u * s * (1.0f + g * (1.0f - s)), dh[q] * a);
        }
        if (r >= left) continue;
        uint4 *dst = reinterpret_cast<uint4 *>(p.dz + (row + r) * (2 * p.N) + 2 * f);
        dst[0] = make_uint4(d[0], d[1], d[2], d[3]);
        dst[1] = make_uint4(d[4], d[5], d[6], d[7]);
        *reinterpret_cast<uint4 *>(static_cast<__nv_bfloat16 *>(p.y) + (row + r) * p.N + f) =
            make_uint4(pack_bf16(h[0], h[1]), pack_bf16(h[2], h[3]), pack_bf16(h[4], h[5]), pack_bf16(h[6], h[7]));
    }
}

// Stages of each of a tile's accumulators.  Where sums are given in fp32 (FINE: the weight gradient) or rounded to 8 bits (the
// gated product), a long sum goes on in another accumulator, and the epilogue adds them up in registers: the tensor core cuts
// off what it adds, up to a unit in the last place with each K = 16 and more where products are 2^10 below the sum.  Gradients of
// mixed signs (norm of the error by the norm; of one sign in brackets) are off by 1.0e-6 (2.2e-6) after 1024 in one accumulator and
// by 1.9e-5 (8.2e-5) after 16384; with 960 at a time by 0.9e-6 (2.0e-6) whatever the length; a chain of fp32 additions by 2e-7 to 4e-7.
// With 1024 at a time one in 25000 of the 8-bit codes falls the other way, whatever the length (one in 3400 with K = 7168 in one
// accumulator; one in 28000 with fp32 additions, and one in 31000 and 115000 with K = 1024).  Shorter pieces keep the epilogue, which
// has to add before it can store, from running under the products: two and three for K of 1024 and 2048 take 15 % more time, 512
// throughout 8-26 %.  A sum that is rounded to bf16 needs no such care.
constexpr int kGradSteps = 960 / kStageK;
template <ExpertOp OP> constexpr int kMostSteps = OP == ExpertOp::kWeightGrad ? kGradSteps : 1024 / kStageK;
template <ExpertOp OP, bool FINE>
__device__ __forceinline__ int acc_steps(int steps)
{
    if (!FINE) return steps;
    const int n = max(1, (steps + kMostSteps<OP> - 1) / kMostSteps<OP>);   // as few pieces as that allows, of equal length
    return (steps + n - 1) / n;
}

// Whether a sum of this call takes more than one accumulator.
template <ExpertOp OP>
__device__ __forceinline__ bool any_split(const KernelParams &p, int lane)
{
    int longest = p.K;
    if (OP == ExpertOp::kWeightGrad) {
        longest = 0;
        for (int s = lane; s < p.P; s += 32) {
            int first;
            longest = max(longest, segment(p, s, first));
        }
        longest = __reduce_max_sync(0xffffffffu, longest);
    }
    return longest > kMostSteps<OP> * kStageK;
}

// 32 features (lanes) x 32 (fp32) or 64 (bf16) columns of a weight gradient, through 4 KB of shared memory: a lane writes
// its feature's 128 bytes, 16-byte units permuted by the feature, and then eight lanes store the 128 bytes of one feature, so
// that whole lines leave and nothing waits.  (By TMA stores the box has to be read before it is filled again, and they queue
// with the loads, which already keep the TMA unit busy: a stage is 256 lines in 512 clocks.  See store_box.)
template <bool F32>
__device__ __forceinline__ void store_grad(const KernelParams &p, const Tile &t, int f, int col, const uint4 (&v)[8], unsigned char *plane,
                                           int lane)
{
#pragma unroll
    for (int q = 0; q < 8; ++q) *reinterpret_cast<uint4 *>(plane + lane * kLine + ((q ^ (lane & 7)) << 4)) = v[q];
    __syncwarp();
    constexpr int kWord = F32 ? 4 : 8;                         // columns of 16 bytes
    const int unit = lane & 7, c = col + unit * kWord;
    char *dst = static_cast<char *>(p.y) + (((size_t)t.slot * p.M + f) * p.N + c) * (16 / kWord);
    const size_t pitch = (size_t)p.N * (16 / kWord);
    const int left = c < p.N ? p.M - f : 0;                    // N is a multiple of 8
#pragma unroll
    for (int half = 0; half < 2; ++half) {                     // four loads on their way at a time
        float4 before[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int r = 16 * half + 4 * i + (lane >> 3);
            if (F32 && p.add && r < left) before[i] = *reinterpret_cast<const float4 *>(dst + r * pitch);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int r = 16 * half + 4 * i + (lane >> 3);
            uint4 o = *reinterpret_cast<const uint4 *>(plane + r * kLine + ((unit ^ (r & 7)) << 4));
            if (F32 && p.add)
                o = make_uint4(__float_as_uint(__uint_as_float(o.x) + before[i].x), __float_as_uint(__uint_as_float(o.y) + before[i].y),
                               __float_as_uint(__uint_as_float(o.z) + before[i].z), __float_as_uint(__uint_as_float(o.w) + before[i].w));
            if (r < left) *reinterpret_cast<uint4 *>(dst + r * pitch) = o;
        }
    }
    __syncwarp();                                              // the plane is free again
}

// The same for 64 columns in bf16 as one TMA store, from a box of 32 lines of 128 bytes with the 128-byte swizzle; what lies
// outside the matrix is cut by the store.  For tiles of few stages, whose stores bound them: the TMA unit has time then, and
// reads the box once where warps would read it and store it (128 slots of 100 rows, 2048 x 4096: 520 us, 585 by the warps; of 511
// rows: 992 and 933).
constexpr int kFewSteps = 4;
__device__ __forceinline__ void store_box(const CUtensorMap *map, int slot, int f, int col, const uint4 (&v)[8], unsigned char *box, int lane)
{
    if (lane == 0) bulk_wait_read<0>();                        // the store before has left the box
    __syncwarp();
#pragma unroll
    for (int q = 0; q < 8; ++q) *reinterpret_cast<uint4 *>(box + lane * kLine + ((q ^ (lane & 7)) << 4)) = v[q];
    fence_async_shared();
    __syncwarp();
    if (lane == 0) {
        asm volatile("cp.async.bulk.tensor.3d.global.shared::cta.tile.bulk_group [%0, {%1, %2, %3}], [%4];" ::"l"(map), "r"(col), "r"(f),
                     "r"(slot), "r"(smem_addr(box))
                     : "memory");
        bulk_commit();
    }
}

// ------------------------------------------------------------------------ kernel

template <ExpertOp OP, bool FINE, bool F32>
__global__ void __launch_bounds__(kThreadsOf<FINE>, 1)
k_expert_product(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b, const __grid_constant__ CUtensorMap map_big,
                 const __grid_constant__ CUtensorMap map_y, const __grid_constant__ ZeroMaps zeros, const KernelParams p)
{
    // map_a: the M operand (weights, or the left operand of a weight gradient); map_b, map_big: the N operand; map_y, zeros: of a
    // weight gradient
    using L = Layout<OP, FINE>;
    constexpr bool kGrad = L::kGrad;
    constexpr int kBox = 32;                                   // rows per TMA load of few rows
    extern __shared__ unsigned char raw[];
    unsigned char *base = reinterpret_cast<unsigned char *>((reinterpret_cast<uintptr_t>(raw) + 1023) & ~(uintptr_t)1023);
    unsigned char *epi = base + L::kEpiOff;
    uint64_t *bars = reinterpret_cast<uint64_t *>(base + L::kBarOff);
    uint64_t *full = bars, *empty = bars + kMaxStages, *tail = bars + 2 * kMaxStages, *peer = bars + 3 * kMaxStages;
    uint64_t *acc_full = bars + 4 * kMaxStages, *acc_empty = acc_full + 2, *drained = acc_full + 4;
    uint32_t *tmem_slot = reinterpret_cast<uint32_t *>(bars + L::kBars);
    volatile int *quit = reinterpret_cast<volatile int *>(tmem_slot + 1);
    int *warp_sums = reinterpret_cast<int *>(tmem_slot + 4), *warp_most = warp_sums + L::kThreads / 32;
    int *ends = reinterpret_cast<int *>(base + L::kEndsOff);
    unsigned char *stage = base + ((L::kEndsOff + (kGrad ? 0 : p.P * 4) + 1023) & ~1023);

    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int rank = (int)cluster_rank();
    if (tid == 0) {
        for (int s = 0; s < kMaxStages; ++s) {
            mbar_init(&full[s], 1); mbar_init(&empty[s], 1);
            mbar_init(&tail[s], 1); mbar_init(&peer[s], 1);
        }
        for (int b = 0; b < 2; ++b) { mbar_init(&acc_full[b], 1); mbar_init(&acc_empty[b], CG * kEpiWarps); }
        mbar_init(drained, 1);
        *quit = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(&map_a));
        asm volatile("prefetch.tensormap [%0];" ::"l"(&map_b));
        if (!kGrad) asm volatile("prefetch.tensormap [%0];" ::"l"(&map_big));
    }
    // hints while the previous kernel drains: its weights have pushed these out of L2 (a hint returns nothing stale)
    if (tid * 32 < p.P) { prefetch_l2(p.slot_counts + tid * 32); prefetch_l2(p.slot_offsets + tid * 32); }
    if (warp == kMmaWarp) tmem_alloc<CG>(tmem_slot, 512);
    __syncwarp();
    tc_fence_before();
    cluster_sync();                                            // the peer's barriers are set up before anything arrives on them
    tc_fence_after();
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");

    int tiles = 0, most_rows = 0;                              // most_rows: of the longest segment
    const int feats = ((kGrad ? p.M : p.N) + CG * kFeat - 1) / (CG * kFeat);
    if (kGrad) {
        tiles = p.P * feats * ((p.N + NT - 1) / NT);           // the host has seen that this is an int
    } else {
        // inclusive prefix over the slots of their tile counts
        const int chunk = (p.P + L::kThreads - 1) / L::kThreads, s0 = tid * chunk, s1 = min(p.P, s0 + chunk);
        int sum = 0, longest = 0;
#pragma unroll 1
        for (int s = s0; s < s1; ++s) {
            int first;
            const int c = segment(p, s, first);
            longest = max(longest, c);
            sum = tiles_sum(sum, feats * row_tiles(c));
            ends[s] = sum;
        }
        longest = __reduce_max_sync(0xffffffffu, longest);
        if (lane == 0) warp_most[warp] = longest;
        int incl = sum;
#pragma unroll 1
        for (int off = 1; off < 32; off <<= 1) {
            const int o = __shfl_up_sync(0xffffffffu, incl, off);
            if (lane >= off) incl = tiles_sum(incl, o);
        }
        if (lane == 31) warp_sums[warp] = incl;
        int before = __shfl_up_sync(0xffffffffu, incl, 1);
        if (lane == 0) before = 0;
        __syncthreads();
        int others = lane < warp ? warp_sums[lane] : 0;        // of the warps before
#pragma unroll
        for (int off = 1; off < 16; off <<= 1) others = tiles_sum(others, __shfl_xor_sync(0xffffffffu, others, off));
        before = tiles_sum(before, __shfl_sync(0xffffffffu, others, 0));
        most_rows = __reduce_max_sync(0xffffffffu, lane < L::kThreads / 32 ? warp_most[lane] : 0);
#pragma unroll 1
        for (int s = s0; s < s1; ++s) ends[s] = tiles_sum(ends[s], before);
        __syncthreads();
    }
    // All 512 columns belong to this CTA, so they start at 0: a constant in every TMEM address.  (Anything else
    // would be reported and no tile touched.)
    constexpr uint32_t tmem = 0;
    const bool whole = *tmem_slot == 0;
    if (tid == 0 && !whole) give_up<CG>(quit);
    if (!kGrad) {
        tiles = ends[p.P - 1];
        // counts that no dispatch writes: nothing is touched
        if (tiles >= kTooManyTiles) {
            if (tid == 0) report_status(p.ctl, kDevCapacity);
            tiles = 0;
        }
    }
    if (!whole) tiles = 0;
    // Where no segment has more than 64 (128) rows, a stage holds 32 (64) of a CTA's and the ring has room for nine (eight)
    // stages and not six: the weights bound the kernel then, and more of them are on their way (one row for 8 slots of
    // 7168 x 2048: gated 97 us instead of 99, down 60 instead of 63).  Weights that run along their features are better off
    // with six (32 slots of 64 rows, 4096 x 2048: gradient by the rows 184 us, with nine 190).
    const int stage_bytes = !L::kAAlongK || most_rows > 128 ? L::kStage : kATile + (most_rows > 64 ? 64 : 32) * kLine;
    const int stages = min(kMaxStages, p.ring / stage_bytes);
    int issued = 0;                                            // stages that this warp has asked for

    if (warp < kEpiWarps) {
        if (FINE) asm volatile("setmaxnreg.inc.sync.aligned.u32 216;");
        // epilogue: TMEM lane = feature of the tile, column = row (weight gradient: column)
        const int group = warp >> 2, quarter = warp & 3;
        unsigned char *mine = epi + warp * L::kEpiWarp;
        constexpr int kPieces = NT / 64;                       // of 32 columns, of this warp: c0 = group * 32, then every 64
        const auto epilogue = [&](auto split) {
            constexpr bool kSplit = decltype(split)::value;
            int buf = 0;
            unsigned acc_parity = 0;
            Tile t;
            bool ok = true;
            for (TileStream<OP> stream(p, ends, tiles); ok && stream.next(t);) {
                const int f = t.feat + rank * kFeat + quarter * 32;
                const int cols = kGrad ? min(NT, p.N - t.col) : t.rows, steps = ((kGrad ? t.rows : p.K) + kStageK - 1) / kStageK;
                const int each = acc_steps<OP, FINE>(steps);
                const auto wait_acc = [&] {
                    // a stage takes 512 clocks, a poll 39 or more: a long sum is no reason to give up
                    ok = __all_sync(0xffffffffu, wait_for(&acc_full[buf], acc_parity, quit, p.spin_limit + 64u * each));
                    tc_fence_after();
                    return ok;
                };
                const auto release_acc = [&] {                     // after this warp's last look at the accumulator
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive_lead<CG>(&acc_empty[buf]);
                };
                const auto next_acc = [&] {
                    buf ^= 1;
                    if (buf == 0) acc_parity ^= 1u;
                };
                const auto acc_at = [&](int c0) { return tmem + buf * NT + c0 + ((uint32_t)(quarter * 32) << 16); };
                uint32_t sum[kSplit ? kPieces : 1][32];
                const auto next_piece = [&] {                      // to the front: a piece's number is no register's
#pragma unroll
                    for (int n = 1; n < kPieces; ++n)
#pragma unroll
                        for (int c = 0; c < 32; ++c) sum[kSplit ? n - 1 : 0][c] = sum[kSplit ? n : 0][c];
                };
                const bool one = !kSplit || each == steps;          // accumulator: its pieces are read as they are stored
                if (!one) {                                        // all of the tile's accumulators added up
                    int k = 0;
#pragma unroll
                    for (int q = 0; q < kPieces; ++q)
#pragma unroll
                        for (int c = 0; c < 32; ++c) sum[q][c] = 0u;
                    do {
                        if (!wait_acc()) break;
#pragma unroll
                        for (int q = 0; q < kPieces; ++q) {
                            if (group * 32 + 64 * q >= cols) break;
                            const uint32_t at = acc_at(group * 32 + 64 * q);
#pragma unroll
                            for (int half = 0; half < 32; half += 16) {
                                uint32_t v[16];
                                if (L::kFragments) tmem_ld_fragment(at + ((uint32_t)half << 16), v);
                                else tmem_ld_lanes(at + half, v);
                                tmem_wait_ld();
#pragma unroll
                                for (int c = 0; c < 16; ++c)
                                    sum[q][half + c] = __float_as_uint(__uint_as_float(sum[q][half + c]) + __uint_as_float(v[c]));
                            }
                        }
                        release_acc();
                        next_acc();
                        k += each;
                    } while (k < steps);
                    if (!ok) break;
                } else if (!wait_acc()) {
                    break;
                }
                if (kGrad && !F32) {
                    for (int c0 = group * 64; c0 < cols && f < p.M; c0 += 128) {
                        uint4 box[8] = {};
                        if (steps > 0) {
                            uint32_t v[2][32];
                            tmem_ld_lanes(acc_at(c0), v[0]);
                            tmem_ld_lanes(acc_at(c0 + 32), v[1]);
                            tmem_wait_ld();
#pragma unroll
                            for (int q = 0; q < 8; ++q) {
                                const uint32_t *w = &v[q >> 2][8 * (q & 3)];
                                box[q] = make_uint4(pack_bf16(__uint_as_float(w[0]), __uint_as_float(w[1])),
                                                    pack_bf16(__uint_as_float(w[2]), __uint_as_float(w[3])),
                                                    pack_bf16(__uint_as_float(w[4]), __uint_as_float(w[5])),
                                                    pack_bf16(__uint_as_float(w[6]), __uint_as_float(w[7])));
                            }
                        }
                        if (steps <= kFewSteps) store_box(&map_y, t.slot, f, t.col + c0, box, mine, lane);
                        else {
                            if (lane == 0) bulk_wait_read<0>();    // of an earlier tile
                            __syncwarp();
                            store_grad<false>(p, t, f, t.col + c0, box, mine, lane);
                        }
                    }
                    release_acc();
                } else if (kGrad) {
#pragma unroll 1
                    for (int q = 0; q < kPieces; ++q) {
                        const int c0 = group * 32 + 64 * q;
                        if (c0 >= cols || f >= p.M || (p.add && steps == 0)) break;
                        if (one && steps > 0) {
                            tmem_ld_lanes(acc_at(c0), sum[0]);
                            tmem_wait_ld();
                        }
                        uint4 box[8];
#pragma unroll
                        for (int i = 0; i < 8; ++i)
                            box[i] = steps > 0 ? make_uint4(sum[0][4 * i], sum[0][4 * i + 1], sum[0][4 * i + 2], sum[0][4 * i + 3]) : make_uint4(0u, 0u, 0u, 0u);
                        store_grad<true>(p, t, f, t.col + c0, box, mine, lane);
                        if (!one) next_piece();
                    }
                    if (one) release_acc();
                } else {
                    float *plane = reinterpret_cast<float *>(mine);
#pragma unroll 1
                    for (int q = 0; q < kPieces; ++q) {
                        const int c0 = group * 32 + 64 * q, left = cols - c0;
                        if (left <= 0) break;
                        const long long row = t.row + c0;
                        Kept kept[4];
                        if (OP == ExpertOp::kGatedBackward) load_kept(p, f, row, left, lane, kept);
                        if (one) {
                            if (L::kFragments) tmem_ld_fragments(acc_at(c0), sum[0]);
                            else tmem_ld_lanes(acc_at(c0), sum[0]);
                            tmem_wait_ld();
                            if (left <= 64) release_acc();
                        }
                        if (!L::kFragments) write_plane(plane, sum[0], lane);
                        if (OP == ExpertOp::kGated) store_gated(p, sum[0], mine, f, row, left, lane);
                        else if (OP == ExpertOp::kGatedBackward) store_gated_backward(p, plane, f, row, left, lane, kept);
                        else store_rows(p, plane, f, row, left, lane);
                        __syncwarp();                              // the plane is free before the next 32 rows are written
                        if (!one) next_piece();
                    }
                    if (one && group * 32 >= cols) release_acc();
                }
                if (one) next_acc();
            }
        };
        // Two epilogues: where every sum is one accumulator's, registers that hold sums would only be in the way (fp32 gradients of
        // 24 slots of 45 rows, 4096 x 1024: 90 us and 119; of 128 slots of 511 rows: 1363 and 1487; gated, 32 slots of 2048 rows, 1024 x
        // 1024, 8-bit sums: 205 and 218).
        if constexpr (FINE) {
            if (any_split<OP>(p, lane)) epilogue(std::true_type());
            else epilogue(std::false_type());
        } else epilogue(std::false_type());
        if (kGrad && !F32 && lane == 0) bulk_wait_all();       // the last stores have left shared memory
    } else {
        // The two issuing warps run their loops with all lanes, so that everything the asynchronous instructions
        // take is uniform over the warp, and issue from one elected lane.
        if (FINE) asm volatile("setmaxnreg.dec.sync.aligned.u32 72;");
        if (warp == kTmaWarp) {
            int s = 0;
            const uint32_t lead = lead_addr<CG>(full);             // the first CTA's barrier counts the bytes of both
            unsigned parity = 1;                                   // a fresh barrier passes the wait for parity 1
            bool ok = true;
            Tile t;
            for (TileStream<OP> stream(p, ends, tiles); ok && stream.next(t);) {
                const int n = tile_n<OP>(p, t), half = n / CG;   // rows (or columns) of the tile in this CTA
                // each TMA instruction costs its warp some 80 cycles: many rows come in one box, few in boxes of 32
                const bool big = half > 2 * kBox;
                const int loads = big ? 1 : (half + kBox - 1) / kBox;
                const uint32_t bytes = CG * (kATile + (kGrad || big ? L::kN : loads * kBox) * kLine);
                const int steps = ((kGrad ? t.rows : p.K) + kStageK - 1) / kStageK;
                const int feat = t.feat + rank * kFeat;
                for (int k = 0; k < steps; ++k) {
                    ok = __all_sync(0xffffffffu, wait_for(&empty[s], parity, quit, p.spin_limit));
                    if (!ok) break;
                    unsigned char *a = stage + s * stage_bytes, *b = a + kATile;
                    if (elect_one()) {
                        uint32_t bar = lead + s * 8;
                        if (kGrad) {
                            const int r = t.row + k * kStageK, col = t.col + rank * half;
                            // a stage whose last lines have to be made zero: the second CTA counts its own bytes
                            const bool own = has_tail(t.rows - k * kStageK);
                            if (rank == 0) mbar_expect_tx(&full[s], own ? bytes / CG : bytes);
                            else if (own) {
                                mbar_expect_tx(&tail[s], bytes / CG);
                                bar = smem_addr(&tail[s]);
                            }
                            if (own) load_grad<false>(a, b, &map_a, &map_b, feat, col, r, bar);
                            else load_grad<true>(a, b, &map_a, &map_b, feat, col, r, bar);
                        } else {
                            if (rank == 0) mbar_expect_tx(&full[s], bytes);
                            if (OP == ExpertOp::kGated) tma_pairs<CG>(a, &map_a, k * kStageK, feat / 16, t.slot, bar);
                            else if (L::kAAlongK) tma_3d<CG>(a, &map_a, k * kStageK, feat, t.slot, bar);
                            else {
#pragma unroll
                                for (int q = 0; q < kFeat / 64; ++q) tma_3d<CG>(a + q * kChunk, &map_a, feat + q * 64, k * kStageK, t.slot, bar);
                            }
                            if (big) tma_2d<CG>(b, &map_big, k * kStageK, t.row + rank * half, bar);
                            else for (int l = 0; l < loads; ++l)
                                tma_2d<CG>(b + l * kBox * kLine, &map_b, k * kStageK, t.row + rank * half + l * kBox, bar);
                        }
                    }
                    __syncwarp();
                    ++issued;
                    if (++s == stages) { s = 0; parity ^= 1u; }
                }
            }
        } else if (warp == kMmaWarp && rank == 0) {
            int s = 0, buf = 0;
            unsigned parity = 0, acc_parity = 1, peer_parity = 0;  // peer_parity: a bit per stage, of its next use
            bool ok = true;
            const uint64_t a_desc = desc_tile<L::kAAlongK>(smem_addr(stage)), b_desc = desc_tile<L::kBAlongK>(smem_addr(stage + kATile));
            Tile t;
            for (TileStream<OP> stream(p, ends, tiles); ok && stream.next(t);) {
                const uint32_t idesc = idesc_bf16<L::kAAlongK, L::kBAlongK>(tile_n<OP>(p, t));
                const int steps = ((kGrad ? t.rows : p.K) + kStageK - 1) / kStageK;
                const int each = acc_steps<OP, FINE>(steps);
                int k = 0;
                do {                                               // once for every accumulator that the tile takes
                    ok = __all_sync(0xffffffffu, wait_for(&acc_empty[buf], acc_parity, quit, p.spin_limit));
                    if (!ok) break;
                    tc_fence_after();
                    const uint32_t d = tmem + buf * NT;
                    const int first = k, last = min(steps, k + each);
                    bool ready = steps > 0 && __all_sync(0xffffffffu, mbar_test_wait(&full[s], parity));
                    for (; k < last; ++k) {
                        if (!ready) {
                            ok = __all_sync(0xffffffffu, wait_for(&full[s], parity, quit, p.spin_limit));
                            if (!ok) break;
                        }
                        // ask for the next stage's barrier now: the answer arrives while this stage is issued
                        const int s_next = s + 1 == stages ? 0 : s + 1;
                        const bool next_full = mbar_test_wait(&full[s_next], s_next ? parity : parity ^ 1u);
                        const int left = t.rows - k * kStageK;     // of a weight gradient
                        if (kGrad && has_tail(left)) {
                            clear_tail(stage + s * stage_bytes, stage_bytes, left, lane);
                            // and the second CTA's
                            if (elect_one()) mbar_expect_tx(&peer[s], (unsigned)(kTailChunks * tail_lines(left) * kLine));
                            __syncwarp();
                            ok = __all_sync(0xffffffffu, wait_for(&peer[s], (peer_parity >> s) & 1u, quit, p.spin_limit));
                            if (!ok) break;
                            peer_parity ^= 1u << s;
                        }
                        tc_fence_after();
                        // descriptors count in 16-byte units
                        const uint64_t a = a_desc + (uint32_t)(s * (stage_bytes >> 4)), b = b_desc + (uint32_t)(s * (stage_bytes >> 4));
                        if (elect_one()) {
#pragma unroll
                            for (int q = 0; q < kStageK / 16; ++q)
                                if (!kGrad || q * 16 < left)
                                    mma_bf16(d, a + q * kDescStep<L::kAAlongK>, b + q * kDescStep<L::kBAlongK>, idesc, k > first || q > 0);
                            mma_commit<CG>(&empty[s]);
                            if (k == last - 1) mma_commit<CG>(&acc_full[buf]);
                        }
                        ready = __all_sync(0xffffffffu, next_full);
                        s = s_next;
                        if (s == 0) parity ^= 1u;
                    }
                    if (!ok) break;
                    if (kGrad && steps == 0 && elect_one()) mma_commit<CG>(&acc_full[buf]);   // nothing to wait for
                    buf ^= 1;
                    if (buf == 0) acc_parity ^= 1u;
                } while (k < steps);
            }
            // everything issued has left the tensor core before TMEM is given back
            if (elect_one()) mma_commit<CG>(drained);
            __syncwarp();
            unsigned long long until = 0;
            drain_wait(drained, 0, until);
        } else if (warp == kMmaWarp && kGrad) {
            // The second CTA of a pair: its share of the stages that end a segment within a K = 16 (see load_zero_tail), once
            // its own bytes of them are there.  (Such a step on every stage: 510 TFLOP/s.)
            int s = 0;
            unsigned tail_parity = 0;                              // a bit per stage, of its next use
            unsigned patience = 0;                                 // a wait begins while the tiles without such an end before it are worked on
            bool ok = true;
            Tile t;
            for (TileStream<OP> stream(p, ends, tiles); ok && stream.next(t);) {
                const int steps = (t.rows + kStageK - 1) / kStageK, left = t.rows - (steps - 1) * kStageK;
                patience = more_patience(patience, p.spin_limit, steps);
                if (steps > 0 && has_tail(left)) {
                    const int at = (s + steps - 1) % stages;
                    ok = __all_sync(0xffffffffu, wait_for(&tail[at], (tail_parity >> at) & 1u, quit, max(p.spin_limit, patience)));
                    if (!ok) break;
                    patience = 0;
                    tail_parity ^= 1u << at;
                    if (elect_one()) load_zero_tail(stage + at * stage_bytes, left, zeros, (int)p.rows, lead_addr<CG>(&peer[at]));
                    __syncwarp();
                }
                s = (s + steps) % stages;
            }
        }
    }

    __syncwarp();
    tc_fence_before();
    cluster_sync();                                            // the pair leaves together: neither arrives on a CTA that is gone
    if (*quit) {                                               // in both CTAs or in none
        // Whichever role gave up, loads may be in flight to this CTA's shared memory, with the first one's barriers: a bounded
        // wait for them before either leaves (the barriers may not complete, but the wait outlasts any copy)
        if (warp == kTmaWarp) {
            unsigned long long until = 0;
            for (int m = max(0, issued - stages); m < issued; ++m) drain_wait(&full[m % stages], (unsigned)(m / stages) & 1u, until);
        }
        __syncwarp();
        cluster_sync();
        if (tid == 0) report_status(p.ctl, kDevTimeout);
    }
    if (warp == kMmaWarp) {
        if (rank == 1) {                                       // the first CTA's last arrival is on its way here as well
            unsigned long long until = 0;
            drain_wait(drained, 0, until);
            __syncwarp();
        }
        tc_fence_after();
        tmem_dealloc<CG>(tmem, 512);
    }
}

// ------------------------------------------------------------------------- host

template <ExpertOp OP, bool FINE = false, bool F32 = false>
cudaError_t launch(const ExpertArgs &a, cudaStream_t st)
{
    using L = Layout<OP, FINE>;
    static_assert(L::kN % 64 == 0 && NT % 32 == 0 && 2 * NT <= 512, "boxes of the row operand, pieces of the epilogue, TMEM columns");
    const auto kernel = k_expert_product<OP, FINE, F32>;
    // a function's attributes are those of one device
    constexpr int kDevices = 64;
    static std::once_flag once[kDevices];
    static cudaError_t attr[kDevices];
    if (a.device < 0 || a.device >= kDevices) return cudaErrorInvalidDevice;
    std::call_once(once[a.device], [&] { attr[a.device] = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, L::kSmem); });
    if (attr[a.device] != cudaSuccess) return attr[a.device];
    if (!encode_fn()) return cudaErrorNotSupported;
    const CUtensorMapDataType bf16 = CU_TENSOR_MAP_DATA_TYPE_BFLOAT16;
    const CUtensorMapSwizzle sw = CU_TENSOR_MAP_SWIZZLE_128B;
    CUtensorMap map_a, map_b, map_big = {}, map_y = {};
    ZeroMaps zeros = {};
    bool ok;
    if (L::kGrad) {
        const cuuint64_t ad[2] = {(cuuint64_t)a.M, (cuuint64_t)a.rows}, as[1] = {2 * (cuuint64_t)a.M};
        const cuuint64_t bd[2] = {(cuuint64_t)a.N, (cuuint64_t)a.rows}, bs[1] = {2 * (cuuint64_t)a.N};
        ok = encode(&map_a, bf16, sw, a.a, 2, ad, as, 64, kStageK) && encode(&map_b, bf16, sw, a.b, 2, bd, bs, 64, kStageK);
        for (int b = 0; b < 4; ++b) ok = ok && encode(&zeros.lines[b], bf16, CU_TENSOR_MAP_SWIZZLE_NONE, a.a, 2, ad, as, 64, 1 << b);
        if (!F32) {
            const cuuint64_t yd[3] = {(cuuint64_t)a.N, (cuuint64_t)a.M, (cuuint64_t)a.P}, ys[2] = {2 * (cuuint64_t)a.N, 2 * (cuuint64_t)a.N * a.M};
            ok = ok && encode(&map_y, bf16, sw, a.y, 3, yd, ys, 64, 32);
        }
    } else {
        const cuuint64_t inner = L::kAAlongK ? a.K : a.N, outer = L::kAAlongK ? a.N : a.K;
        const cuuint64_t wd[3] = {inner, outer, (cuuint64_t)a.P}, ws[2] = {2 * inner, 2 * inner * outer};
        const cuuint64_t ad[2] = {(cuuint64_t)a.K, (cuuint64_t)a.rows}, as[1] = {2 * (cuuint64_t)a.K};
        // a row, eight rows of one parity, the parities, the sixteens, the slots
        const cuuint64_t pd[5] = {(cuuint64_t)a.K, 8, 2, (cuuint64_t)a.N / 16, (cuuint64_t)a.P};
        const cuuint64_t ps[4] = {4 * (cuuint64_t)a.K, 2 * (cuuint64_t)a.K, 32 * (cuuint64_t)a.K, 2 * (cuuint64_t)a.K * a.N};
        ok = (OP == ExpertOp::kGated ? encode(&map_a, bf16, sw, a.w, 5, pd, ps, 64, 8, 2, kFeat / 16)
                                     : encode(&map_a, bf16, sw, a.w, 3, wd, ws, 64, L::kAAlongK ? kFeat : kStageK)) &&
             encode(&map_b, bf16, sw, a.a, 2, ad, as, 64, 32) &&
             encode(&map_big, bf16, sw, a.a, 2, ad, as, 64, L::kN);
    }
    if (!ok) return cudaErrorInvalidValue;
    KernelParams p;
    p.slot_counts = a.slot_counts; p.slot_offsets = a.slot_offsets; p.rows = a.rows;
    p.P = a.P; p.N = a.N; p.K = a.K; p.M = a.M; p.ring = L::ring(a.P);
    p.y = a.y; p.z = a.z; p.z_scales = a.z_scales; p.dz = static_cast<__nv_bfloat16 *>(a.dz);
    p.add = a.add; p.ctl = a.ctl; p.spin_limit = a.spin_limit;
    // no more CTAs than there can be tiles (the counts are on the device)
    const long long feats = ((L::kGrad ? a.M : a.N) + CG * kFeat - 1) / (CG * kFeat);
    const long long most = L::kGrad ? feats * ((a.N + NT - 1) / NT) * a.P : feats * (std::min<long long>(a.P, a.rows) + a.rows / NT);
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(CG * std::min<long long>(a.sm_count / CG, most)));
    cfg.blockDim = dim3(L::kThreads); cfg.dynamicSmemBytes = L::bytes(a.P); cfg.stream = st;
    cudaLaunchAttribute at[2];
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim.x = CG; at[0].val.clusterDim.y = 1; at[0].val.clusterDim.z = 1;
    at[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = at; cfg.numAttrs = a.pdl ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, kernel, map_a, map_b, map_big, map_y, zeros, p);
}

}  // namespace

namespace moe {

cudaError_t expert_product_launch(const ExpertArgs &a, cudaStream_t st)
{
    switch (a.op) {
    case ExpertOp::kProduct: return launch<ExpertOp::kProduct>(a, st);
    case ExpertOp::kGated: return launch<ExpertOp::kGated, true>(a, st);      // its output does not depend on what is kept
    case ExpertOp::kTransposed: return launch<ExpertOp::kTransposed>(a, st);
    case ExpertOp::kGatedBackward: return launch<ExpertOp::kGatedBackward>(a, st);
    case ExpertOp::kWeightGrad:
        if (!a.f32) return launch<ExpertOp::kWeightGrad>(a, st);
        // no segment is longer than the buffer: one accumulator will do, without a look at the segments (2 % of 24 slots of 45 rows,
        // 4096 x 1024)
        if (a.rows <= kGradSteps * kStageK) return launch<ExpertOp::kWeightGrad, false, true>(a, st);
        return launch<ExpertOp::kWeightGrad, true, true>(a, st);
    }
    return cudaErrorInvalidValue;
}

}  // namespace moe
