// The experts' products on 4-bit rows: for every physical slot p and every row r of its segment
//     out[r, f] = sum_k a[r, k] * w[p, f, k]          (fp32 accumulation on the tensor cores)
// with both operands microscaled (mx_format.cuh), on tcgen05.mma kind::mxf4 with block scales: the
// scales are applied inside the tensor core, nothing is unpacked.
//
// Weights are the M operand (128 features of one slot per tile) and rows the N operand, so a segment
// of any length costs N = its length rounded up to 16, from one token to hundreds, and a tile's
// accumulator is [128 lanes = features] x [columns = rows] in TMEM.  K goes in stages of 256 (128
// bytes of a code row: one 128-byte swizzle span, four MMAs of K = 64).
//
// One persistent CTA per SM:
//   warps 0-7   epilogue, two groups of four (a warp reads one quarter of the TMEM lanes): TMEM -> registers ->
//               shared memory -> HBM, 32 rows at a time, the groups taking turns
//   warp 8      TMA loads of the code tiles (weights 128 x 128 B, rows n x 128 B, 128-byte swizzle)
//   warp 9      scales shared -> TMEM (tcgen05.cp) and the MMAs, from one thread
//   warps 10-   scales, two warps per 128 rows: HBM -> registers -> the 32 x 16-byte blocks tcgen05.cp wants
// The accumulator is double buffered, so the epilogue of a tile runs under the products of the next.
//
// Tiles are dealt feature tile by feature tile of a slot, row tile innermost: CTAs that work at the same time
// share a weight tile (through L2) as often as possible.  How slots are ordered: see Order.
#include "mx_product.h"

#include <algorithm>
#include <mutex>

#include "mx_format.cuh"
#include "tcgen05.cuh"

namespace {

using namespace moe;

constexpr int kFeat = 128;                 // features per CTA and tile
constexpr int kStageK = 256;               // elements of K per stage
constexpr int kRowBytes = kStageK / 2;     // bytes of a code row per stage
constexpr int kATile = kFeat * kRowBytes;  // 16 KB
constexpr int kMaxP = 4096, kFullTableP = kMaxP / 4;   // slots up to which the tables of Order fit in full
constexpr int kEpiWarps = 8, kTmaWarp = kEpiWarps, kMmaWarp = kEpiWarps + 1, kScaleWarp = kEpiWarps + 2;

// ------------------------------------------------------------------ tcgen05 in PTX (the rest: tcgen05.cuh)

template <int CG>
__device__ __forceinline__ void mma_mxf4(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t sfa, uint32_t sfb, bool accumulate)
{
    if (CG == 1)
        asm volatile(
            "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %6, 0;\n\t"
            "tcgen05.mma.cta_group::1.kind::mxf4.block_scale.scale_vec::2X [%0], %1, %2, %3, [%4], [%5], p;\n\t}" ::"r"(d),
            "l"(a), "l"(b), "r"(idesc), "r"(sfa), "r"(sfb), "r"((uint32_t)accumulate)
            : "memory");
    else
        asm volatile(
            "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %6, 0;\n\t"
            "tcgen05.mma.cta_group::2.kind::mxf4.block_scale.scale_vec::2X [%0], %1, %2, %3, [%4], [%5], p;\n\t}" ::"r"(d),
            "l"(a), "l"(b), "r"(idesc), "r"(sfa), "r"(sfb), "r"((uint32_t)accumulate)
            : "memory");
}

// 32 rows of 16 bytes from shared memory to four TMEM columns, repeated in the four lane quarters (with
// CG = 2 in both CTAs, each from its own shared memory)
template <int CG>
__device__ __forceinline__ void cp_scales(uint32_t tmem, uint64_t desc)
{
    if (CG == 1) asm volatile("tcgen05.cp.cta_group::1.32x128b.warpx4 [%0], %1;" ::"r"(tmem), "l"(desc) : "memory");
    else asm volatile("tcgen05.cp.cta_group::2.32x128b.warpx4 [%0], %1;" ::"r"(tmem), "l"(desc) : "memory");
}

// Shared-memory matrix descriptor: start and strides in 16-byte units, version 1 (sm_100).
// Code tiles: K-major, 128-byte swizzle, 8-row groups 1024 bytes apart.
// Scale blocks: no swizzle, 8-row groups (8 x 16 bytes) 128 bytes apart.
__device__ __forceinline__ uint64_t desc_codes(uint32_t addr)
{
    return (uint64_t)((addr >> 4) & 0x3fffu) | (1ull << 16) | (64ull << 32) | (1ull << 46) | (2ull << 61);
}
__device__ __forceinline__ uint64_t desc_scales(uint32_t addr)
{
    return (uint64_t)((addr >> 4) & 0x3fffu) | (1ull << 16) | (8ull << 32) | (1ull << 46);
}

// Instruction descriptor of kind::mxf4: A and B e2m1 (1), both K-major, scales ue8m0 (bit 23),
// N / 8 at bit 17, M / 16 at bit 24; sf_half: which half of a 32-bit scale word (0 or 2) belongs to this K = 64.
template <int CG>
__device__ __forceinline__ uint32_t idesc_mxf4(int n)
{
    return (1u << 7) | (1u << 10) | ((uint32_t)(n >> 3) << 17) | (1u << 23) | ((uint32_t)(CG * kFeat >> 4) << 24);
}
__device__ __forceinline__ constexpr uint32_t sf_half(uint32_t id) { return (id << 4) | (id << 29); }

// ------------------------------------------------------------------------ tiles

struct KernelParams {
    const uint8_t *a_scales, *w_scales;
    const int32_t *slot_counts, *slot_offsets;
    long long rows;
    int P, N, K;
    __nv_bfloat16 *y;
    uint8_t *h_codes, *h_scales;
    Control *ctl;
    unsigned spin_limit;
};

struct Tile {
    int slot, feat;        // slot, first feature
    int row;               // first row
    int rows;              // rows of the tile (1 .. NT)
    __device__ int n() const { return (rows + 15) & ~15; }
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
template <int NT>
__device__ __forceinline__ int row_tiles(int c) { return (c + NT - 1) / NT; }

// The order of the tiles.  A slot whose rows fit one tile is bound by its weights (HBM), one with several row tiles by
// the products (its weights come from L2 after the first), and neighbours in the order run at the same time.  So the
// tiles of both kinds are merged in proportion, each kind in its own order, instead of slot by slot: with a popularity
// skew HBM then works all the time and not in turn with the tensor cores.  (Everything here is kept short: between
// two launches the weights push this code out of L2, and in a call of 20 us every line of it is fetched anew.)
struct Order {
    const int *many, *one;     // inclusive prefix over the slots of the tiles of either kind
    const int2 *segments;      // first row and rows of every slot; NULL = read them again
    unsigned share;            // 2^32 * (tiles of the first kind) / (all tiles), rounded up; 0 = all are of the second
};

template <int NT, int CG>
__device__ __forceinline__ Tile tile_at(const KernelParams &p, const Order &o, int index)
{
    const int *ends = o.one;
    if (o.share) {                                   // tiles before `index` that are of the first kind, and whether this one is
        const int m = (int)__umulhi(index, o.share), m1 = (int)__umulhi(index + 1, o.share);
        if (m1 > m) ends = o.many;
        index = m1 > m ? m : index - m;
    }
    int lo = 0, hi = p.P - 1;                        // first slot whose inclusive end is beyond the index
#pragma unroll 1
    while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if (ends[mid] > index) hi = mid; else lo = mid + 1;
    }
    const int local = index - (lo ? ends[lo - 1] : 0);
    Tile t;
    int first, c;
    if (o.segments) { const int2 sg = o.segments[lo]; first = sg.x; c = sg.y; }
    else c = segment(p, lo, first);
    const int nt = row_tiles<NT>(c);
    const int f = local / nt, r = local - f * nt;
    const int size = ((c + nt - 1) / nt + 31) & ~31;
    t.slot = lo; t.feat = f * (CG * kFeat);
    t.row = first + r * size;
    t.rows = min(size, c - r * size);                // may be <= 0 for the last tile of an uneven cut
    return t;
}

// Shared memory of the epilogue: a box of bf16 rows per pair of warps (store_plain) or two planes of fp32 per group
// of four (store_gated); twice, used in turn, where many rows make the epilogue as long as the products.
constexpr int kPlane = 32 * 32 + 8, kPlaneBytes = (2 * kPlane * 4 + 127) / 128 * 128, kBoxBytes = 4096;

// The tiles of a CTA (or pair of CTAs) of a grid of `step`, first, first + step, ..., as a warp sees them.  Finding a
// tile is a chain of dependent reads, so the lanes find the next 32 of them side by side and hand them out one by one.
template <int NT, int CG>
struct TileStream {
    const KernelParams &p;
    const Order &o;
    const int tiles;
    int base, at;
    Tile mine;
    __device__ TileStream(const KernelParams &p_, const Order &o_, int tiles_)
        : p(p_), o(o_), tiles(tiles_), base(blockIdx.x / CG), at(32), mine{}
    {
    }
    __device__ bool next(Tile &t)                    // false when there are no more
    {
        while (true) {
            if (at == 32) {
                if (base >= tiles) return false;
                const int step = (int)gridDim.x / CG, i = base + (int)(threadIdx.x & 31) * step;
                mine.rows = 0; mine.slot = -1;
                if (i < tiles) mine = tile_at<NT, CG>(p, o, i);
                base += 32 * step;
                at = 0;
                __syncwarp();
            }
            t.slot = __shfl_sync(0xffffffffu, mine.slot, at); t.feat = __shfl_sync(0xffffffffu, mine.feat, at);
            t.row = __shfl_sync(0xffffffffu, mine.row, at); t.rows = __shfl_sync(0xffffffffu, mine.rows, at);
            ++at;
            if (t.slot < 0) return false;
            if (t.rows > 0) return true;
        }
    }
};

// The next tile with its fields and the verdict in uniform registers (a warp reduction writes those): what
// tcgen05 and TMA instructions take comes from uniform registers, and a value or a loop that the compiler
// cannot prove uniform costs a move per operand and instruction.
template <int NT, int CG>
__device__ __forceinline__ bool next_uniform(TileStream<NT, CG> &stream, Tile &t)
{
    Tile m;
    const bool more = stream.next(m);
    if (!__any_sync(0xffffffffu, more)) return false;
    t.slot = (int)__reduce_max_sync(0xffffffffu, (unsigned)m.slot); t.feat = (int)__reduce_max_sync(0xffffffffu, (unsigned)m.feat);
    t.row = (int)__reduce_max_sync(0xffffffffu, (unsigned)m.row); t.rows = (int)__reduce_max_sync(0xffffffffu, (unsigned)m.rows);
    return true;
}

// Row of a gated tile's weights that lies at place r: of each sixteen first the even rows (gates), then the odd ones
// (up-projections)
__device__ __forceinline__ int weight_row(int r) { return (r & ~15) + 2 * (r & 7) + ((r >> 3) & 1); }

template <int NT, int STAGES, int CG, bool GATED>
struct Layout {
    static constexpr int kBTile = (NT / CG + 31) / 32 * 32 * kRowBytes;   // this CTA's rows, in boxes of 32
    static constexpr int kRB = (NT + 127) / 128;              // 128-row scale blocks of the row operand
    static constexpr int kThreads = 32 * (kEpiWarps + 2 + 2 * (1 + kRB));
    static constexpr int kSfA = 2 * 512, kSfB = 2 * kRB * 512;
    static constexpr int kStage = kATile + kBTile;            // multiples of 1024: swizzle alignment
    static constexpr int kSf = kSfA + kSfB;
    static constexpr int kStageOff = 0;
    static constexpr int kSfOff = STAGES * kStage;
    static constexpr int kEpiOff = kSfOff + STAGES * kSf;
    static constexpr int kEpiBufs = NT > 64 ? 2 : 1, kEpiBuf = GATED ? kPlaneBytes : 2 * kBoxBytes;
    static constexpr int kEpiBytes = 2 * kEpiBufs * kEpiBuf;
    static constexpr int kBarOff = kEpiOff + kEpiBytes;
    static constexpr int kBars = 2 * STAGES + 5;
    static constexpr int kEndsOff = kBarOff + ((kBars * 8 + 32 + 15) & ~15);
    static size_t bytes(int P) { return 1024 + kEndsOff + (size_t)P * (P <= kFullTableP ? 16 : 4); }
};

// Bounded wait.  `quit` is shared by the CTA: the first role that gives up sets it (in both CTAs of a pair), the others follow.
template <int CG>
__device__ __forceinline__ bool wait_for(uint64_t *bar, unsigned parity, volatile int *quit, unsigned limit)
{
    unsigned spins = 0;
    while (!mbar_try_wait(bar, parity)) {
        if (++spins > limit || ((spins & 63u) == 0 && *quit)) { give_up<CG>(quit); return false; }
    }
    return true;
}

// ---------------------------------------------------------------------- epilogue

// Verdict of the warps that share a barrier: true if it is true for all of them.
__device__ __forceinline__ bool warps_all(int barrier, int threads, bool ok)
{
    uint32_t r;
    asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.u32 p, %1, 0;\n\tbarrier.cta.red.and.pred q, %2, %3, p;\n\tselp.u32 %0, 1, 0, q;\n\t}"
                 : "=r"(r) : "r"((uint32_t)ok), "r"(barrier), "r"(threads) : "memory");
    return r != 0;
}

__device__ __forceinline__ void group_sync(int group) { asm volatile("barrier.cta.sync %0, 128;" ::"r"(group + 1) : "memory"); }

__device__ __forceinline__ void pair_sync(int pair) { asm volatile("barrier.cta.sync %0, 64;" ::"r"(pair + 1) : "memory"); }

// 64 features (two warps) x 32 rows of the accumulator as bf16 rows, through 4 KB of shared memory: a box of
// [32 rows][64 features], 128-byte swizzle.  The accumulator is read in the fragment layout (lane / 4 = feature, two
// neighbouring rows per register pair), so that a pair is one bf16x2 and stmatrix writes it transposed.  32 rows
// that all belong to the segment leave as a TMA store, which costs the warps nothing; the last rows of a segment leave
// as 16-byte stores, so that the rows behind it stay as they are.  (Every load or store of these warps has to queue
// for the shared memory that the products keep busy, and warps that wait for one another wait for the slowest: boxes
// of four warps were 10 % slower with short K.  Boxes of one warp, 64 bytes to a row, cost 8 % in L2 with long rows.)
// The fp32 sum is rounded once.
template <int BUFS>
__device__ __forceinline__ void store_plain(const KernelParams &p, const CUtensorMap *map_y, const Tile &t, int c0, const uint32_t (&v)[32],
                                            unsigned char *buf, int pair, int half, int lane)
{
    const uint32_t base = smem_addr(buf);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        uint32_t m[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) {                          // features 8q .. 8q + 7 of the warp's 32
            const int at = (q >> 1) * 16 + 4 * i + (q & 1) * 2;
            const __nv_bfloat162 h = __floats2bfloat162_rn(__uint_as_float(v[at]), __uint_as_float(v[at + 1]));
            m[q] = *reinterpret_cast<const uint32_t *>(&h);
        }
        const int r = 8 * i + (lane & 7), piece = half * 4 + (lane >> 3);   // this lane's row and 16-byte piece
        asm volatile("stmatrix.sync.aligned.m8n8.x4.trans.shared.b16 [%0], {%1, %2, %3, %4};" ::"r"(base + r * 128 + ((piece ^ (r & 7)) << 4)),
                     "r"(m[0]), "r"(m[1]), "r"(m[2]), "r"(m[3])
                     : "memory");
    }
    fence_async_shared();
    const bool leader = half == 0 && lane == 0;
    if (leader && BUFS == 2) bulk_wait_read<0>();              // the other buffer's store has left it
    pair_sync(pair);
    const int left = t.rows - c0, f = t.feat + (pair & 1) * 64;
    if (left >= 32) {
        if (leader && f < p.N) {
            asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.tile.bulk_group [%0, {%1, %2}], [%3];" ::"l"(map_y), "r"(f),
                         "r"(t.row + c0), "r"(base)
                         : "memory");
            bulk_commit();
        }
    } else {
        const int tid = half * 32 + lane, piece = tid & 7;
        uint4 o[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int r = (tid >> 3) + 8 * i;
            o[i] = *reinterpret_cast<const uint4 *>(buf + r * 128 + ((piece ^ (r & 7)) << 4));
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int r = (tid >> 3) + 8 * i;
            if (r < left && f + piece * 8 < p.N) *reinterpret_cast<uint4 *>(p.y + (size_t)(t.row + c0 + r) * p.N + f + piece * 8) = o[i];
        }
    }
    if (BUFS == 1) {                                           // one buffer: free before the next 32 rows are written
        if (leader) bulk_wait_read<0>();
        pair_sync(pair);
    }
}

__device__ __forceinline__ float silu(float g)
{
    // Both flush to zero: below g = -87.3, where the sigmoid is less than 2^-126, the result is 0.  (The formula in 32
    // bits does the same from g = -88.7 on, where exp overflows.)
    float e, r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(g * -1.44269504f));
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(1.0f + e));
    return g * r;
}

// SwiGLU and quantisation of 128 weight rows (64 pairs of a gate and its up-projection) x 32 rows.  The weight rows of
// a sixteen lie in the order of weight_row, so that the fragment layout gives a thread both halves of its pairs: of
// feature lane / 4 (and 8 more) for the rows 8 j + 2 (lane % 4) and one more.  The 64 results of a row then go through
// shared memory, two planes (blocks of 32 features) of [32 rows][32], where each half block is taken by one thread and
// the block's largest magnitude by one shuffle.  In a plane the eights of a row are swapped by row / 2 % 4 and their
// fours by row % 2: no two lanes of a store or of a load of 16 bytes meet in a bank.  (Weight rows in their own
// order, pairs in neighbouring lanes that trade a value by shuffle: 73.4 us instead of 71.4 for 4096 rows over 8 experts
// of 4096 x 4096, 711 instead of 706 for 65536 over 16 of 7168 x 2048.)  Everything before the one rounding to 4 bits
// is fp32; exp and the reciprocal are the hardware's approximations (2 and 1 units in the last place), and the rounded
// argument of exp costs up to |g| 2^-24 relative besides, all far below a 4-bit step.
__device__ __forceinline__ void store_gated(const KernelParams &p, const Tile &t, int c0, const uint32_t (&v)[32], float *buf,
                                            int group, int quarter, int lane)
{
    float *w = buf + (quarter >> 1) * kPlane + (lane & 3) * 64;
#pragma unroll
    for (int e = 0; e < 2; ++e) {
        const int eight = (((quarter & 1) * 2 + e) ^ (lane & 3)) * 8;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            float *at = w + i * 32 + eight + ((lane >> 2) ^ (4 * i));
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float gate = __uint_as_float(v[16 * e + 4 * j + i]), up = __uint_as_float(v[16 * e + 4 * j + 2 + i]);
                at[256 * j] = silu(gate) * up;
            }
        }
    }
    group_sync(group);
    const int tid = quarter * 32 + lane, r = tid >> 2, blk = (tid >> 1) & 1, half = tid & 1;
    const float *src = buf + blk * kPlane + r * 32;
    const int swap = (half * 16) ^ (((r >> 1) & 3) * 8) ^ ((r & 1) * 4);
    float x[2][8];
    uint32_t a = 0;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        const float4 f = *reinterpret_cast<const float4 *>(src + (swap ^ (4 * q)));
        const float e[4] = {f.x, f.y, f.z, f.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[q >> 1][(q & 1) * 4 + i] = e[i];
            a = max(a, __float_as_uint(e[i]) & 0x7fffffffu);
        }
    }
    a = max(a, __shfl_xor_sync(0xffffffffu, a, 1));
    const uint32_t s = mx_scale_byte(a);
    const float inv = mx_inverse_scale(s);
    uint32_t c[2];
#pragma unroll
    for (int q = 0; q < 2; ++q) {
#pragma unroll
        for (int i = 0; i < 8; ++i) x[q][i] *= inv;
        c[q] = s == 255u ? 0u : mx_pack8(x[q]);
    }
    const int cols = p.N / 2, h = t.feat / 2 + blk * 32;       // first feature of the block
    if (c0 + r < t.rows && h < cols) {
        const size_t row = (size_t)(t.row + c0 + r);
        *reinterpret_cast<uint2 *>(p.h_codes + row * (cols / 2) + h / 2 + half * 8) = make_uint2(c[0], c[1]);
        if (half == 0) p.h_scales[row * mx_scale_pitch(cols) + h / kMxBlock] = (uint8_t)s;
    }
}

template <int NT, int STAGES, int CG, bool GATED>
__global__ void __launch_bounds__(Layout<NT, STAGES, CG, GATED>::kThreads, 1)
k_mx_product(const __grid_constant__ CUtensorMap map_w, const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_big,
             const __grid_constant__ CUtensorMap map_y, const KernelParams p)
{
    using L = Layout<NT, STAGES, CG, GATED>;
    constexpr int kBox = 32, kBig = NT / CG;                   // rows per TMA load of the row operand
    extern __shared__ unsigned char raw[];
    unsigned char *base = reinterpret_cast<unsigned char *>((reinterpret_cast<uintptr_t>(raw) + 1023) & ~(uintptr_t)1023);
    unsigned char *stage = base + L::kStageOff, *sf = base + L::kSfOff, *epi = base + L::kEpiOff;
    uint64_t *bars = reinterpret_cast<uint64_t *>(base + L::kBarOff);
    uint64_t *full = bars, *empty = bars + STAGES;
    uint64_t *acc_full = bars + 2 * STAGES, *acc_empty = acc_full + 2, *drained = acc_full + 4;
    uint32_t *tmem_slot = reinterpret_cast<uint32_t *>(bars + L::kBars);
    volatile int *quit = reinterpret_cast<volatile int *>(tmem_slot + 1);
    int *warp_sums = reinterpret_cast<int *>(epi);             // free before the first epilogue
    int *ends = reinterpret_cast<int *>(base + L::kEndsOff);

    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int rank = CG == 2 ? (int)cluster_rank() : 0;
    if (tid == 0) {
        for (int s = 0; s < STAGES; ++s) {
            mbar_init(&full[s], 1 + CG * (1 + L::kRB));        // the bytes of the loads, and every scale warp of the pair
            mbar_init(&empty[s], 1);
        }
        for (int b = 0; b < 2; ++b) { mbar_init(&acc_full[b], 1); mbar_init(&acc_empty[b], CG * kEpiWarps); }
        mbar_init(drained, 1);
        *quit = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(&map_w));
        asm volatile("prefetch.tensormap [%0];" ::"l"(&map_a));
        asm volatile("prefetch.tensormap [%0];" ::"l"(&map_big));
        if (!GATED) asm volatile("prefetch.tensormap [%0];" ::"l"(&map_y));
    }
    // hints while the previous kernel drains: its weights have pushed these out of L2 (a hint returns nothing stale)
    if (tid * 32 < p.P) { prefetch_l2(p.slot_counts + tid * 32); prefetch_l2(p.slot_offsets + tid * 32); }
    if (warp == kMmaWarp) tmem_alloc<CG>(tmem_slot, 512);
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");

    // inclusive prefixes over the slots of their tile counts: with up to kFullTableP slots for both kinds (see
    // Order), and the segments beside them, with more all slots as one kind
    const int feats = (p.N + CG * kFeat - 1) / (CG * kFeat);
    const bool merge = p.P <= kFullTableP;
    int2 *segments = reinterpret_cast<int2 *>(ends);           // with the full tables: [P] segments, [P] many, [P] one
    int *many = ends + 2 * p.P;
    if (merge) ends += 3 * p.P;
    {
        const int chunk = (p.P + L::kThreads - 1) / L::kThreads;
        const int s0 = tid * chunk, s1 = min(p.P, s0 + chunk);
        int sum[2] = {0, 0};
#pragma unroll 1
        for (int s = s0; s < s1; ++s) {
            int first;
            const int c = segment(p, s, first), nt = row_tiles<NT>(c);
            if (merge) segments[s] = make_int2(first, c);
            if (merge && nt > 1) sum[1] = tiles_sum(sum[1], feats * nt);
            else sum[0] = tiles_sum(sum[0], feats * nt);
            ends[s] = sum[0];
            if (merge) many[s] = sum[1];
        }
        int before[2];
#pragma unroll
        for (int q = 0; q < 2; ++q) {                          // (loops that are run once are not unrolled)
            int incl = sum[q];
#pragma unroll 1
            for (int off = 1; off < 32; off <<= 1) {
                const int o = __shfl_up_sync(0xffffffffu, incl, off);
                if (lane >= off) incl = tiles_sum(incl, o);
            }
            if (lane == 31) warp_sums[2 * warp + q] = incl;
            before[q] = __shfl_up_sync(0xffffffffu, incl, 1);
            if (lane == 0) before[q] = 0;
        }
        __syncthreads();
#pragma unroll 1
        for (int w = 0; w < warp; ++w) {
            before[0] = tiles_sum(before[0], warp_sums[2 * w]); before[1] = tiles_sum(before[1], warp_sums[2 * w + 1]);
        }
#pragma unroll 1
        for (int s = s0; s < s1; ++s) {
            ends[s] = tiles_sum(ends[s], before[0]);
            if (merge) many[s] = tiles_sum(many[s], before[1]);
        }
    }
    __syncwarp();
    tc_fence_before();
    if (CG == 2) cluster_sync();                               // the peer's barriers are set up before anything arrives on them
    else __syncthreads();
    tc_fence_after();
    // All 512 columns belong to this CTA, so they start at 0: a constant in every TMEM address.  (Anything else
    // would be reported and no tile touched.)
    constexpr uint32_t tmem = 0;
    const bool whole = *tmem_slot == 0;
    if (tid == 0 && !whole) give_up<CG>(quit);
    const int n_many = merge ? many[p.P - 1] : 0, n_all = tiles_sum(ends[p.P - 1], n_many);
    Order order = {many, ends, merge ? segments : nullptr, 0u};
    if (n_many == n_all) order.one = many;                     // only that kind
    // share * n_all / 2^32 is n_many and a fraction: exactly n_many of the n_all tiles are of the first kind
    else if (n_many > 0) order.share = (unsigned)(((unsigned long long)n_many << 32) / (unsigned)n_all) + 1u;
    const bool sane = n_all < kTooManyTiles;                   // else counts that no dispatch writes: nothing is touched
    if (tid == 0 && !sane) report_status(p.ctl, kDevCapacity);
    const int tiles = whole && sane ? n_all : 0;
    const int steps = (p.K + kStageK - 1) / kStageK;
    constexpr uint32_t kSfCol = 2 * NT;                        // scale columns follow the two accumulators
    constexpr uint32_t kSfaCols = 8, kSfbCols = 8 * L::kRB;    // per stage parity
    static_assert(2 * NT + 2 * (kSfaCols + kSfbCols) <= 512, "TMEM columns");

    // The two issuing warps run their loops with all lanes, so that everything the asynchronous instructions
    // take is uniform over the warp, and issue from one elected lane.  (Behind a plain `lane == 0` the
    // compiler cannot know that one lane is left and serialises every such instruction over the warp: 80
    // cycles each, 700-1300 per stage, which bound the whole kernel.)
    int issued = 0;                                            // stages that this warp has asked for
    if (warp == kTmaWarp) {
        int s = 0;
        const uint32_t lead = lead_addr<CG>(full);
        unsigned parity = 1;                                   // a fresh barrier passes the wait for parity 1
        bool ok = true;
        Tile t;
        for (TileStream<NT, CG> stream(p, order, tiles); ok && next_uniform(stream, t);) {
            const int half = t.n() / CG;                       // rows of the tile in this CTA
            // each TMA instruction costs its warp some 80 cycles: many rows come in one box, few in boxes of 32
            const bool big = half > 2 * kBox;
            const int loads = big ? 1 : (half + kBox - 1) / kBox;
            const uint32_t bytes = CG * (kATile + (big ? kBig : loads * kBox) * kRowBytes);
            for (int k = 0; k < steps; ++k) {
                ok = __all_sync(0xffffffffu, wait_for<CG>(&empty[s], parity, quit, p.spin_limit));
                if (!ok) break;
                unsigned char *a = stage + s * L::kStage, *b = a + kATile;
                if (elect_one()) {
                    // the first CTA's barrier counts the bytes of both
                    if (rank == 0) mbar_expect_tx(&full[s], bytes);
                    const uint32_t bar = lead + s * 8;
                    if (GATED) tma_pairs<CG>(a, &map_w, k * kRowBytes, (t.feat + rank * kFeat) / 16, t.slot, bar);
                    else tma_3d<CG>(a, &map_w, k * kRowBytes, t.feat + rank * kFeat, t.slot, bar);
                    if (big) tma_2d<CG>(b, &map_big, k * kRowBytes, t.row + rank * half, bar);
                    else for (int l = 0; l < loads; ++l)
                        tma_2d<CG>(b + l * kBox * kRowBytes, &map_a, k * kRowBytes, t.row + rank * half + l * kBox, bar);
                }
                __syncwarp();
                ++issued;
                if (++s == STAGES) { s = 0; parity ^= 1u; }
            }
        }
    } else if (warp == kMmaWarp && rank == 0) {
        int s = 0, buf = 0;
        unsigned parity = 0, acc_parity = 1, step_no = 0;
        bool ok = true;
        const uint64_t stage_desc = desc_codes(smem_addr(stage)), sf_desc = desc_scales(smem_addr(sf));
        Tile t;
        for (TileStream<NT, CG> stream(p, order, tiles); ok && next_uniform(stream, t);) {
            ok = __all_sync(0xffffffffu, wait_for<CG>(&acc_empty[buf], acc_parity, quit, p.spin_limit));
            if (!ok) break;
            tc_fence_after();
            const uint32_t d = tmem + buf * NT;
            const int n = t.n();
            const uint32_t idesc = idesc_mxf4<CG>(n);
            bool ready = __all_sync(0xffffffffu, mbar_test_wait(&full[s], parity));
            for (int k = 0; k < steps; ++k, ++step_no) {
                if (!ready) {
                    ok = __all_sync(0xffffffffu, wait_for<CG>(&full[s], parity, quit, p.spin_limit));
                    if (!ok) break;
                }
                tc_fence_after();
                // ask for the next stage's barrier now: the answer arrives while this stage is issued
                const int s_next = s + 1 == STAGES ? 0 : s + 1;
                const bool next_full = mbar_test_wait(&full[s_next], s_next ? parity : parity ^ 1u);
                // descriptors count in 16-byte units
                const uint64_t a = stage_desc + (uint32_t)(s * (L::kStage >> 4)), b = a + (kATile >> 4);
                const uint64_t sfs = sf_desc + (uint32_t)(s * (L::kSf >> 4));
                const uint32_t sfa = tmem + kSfCol + (step_no & 1) * (kSfaCols + kSfbCols), sfb = sfa + kSfaCols;
                if (elect_one()) {
#pragma unroll
                    for (int g = 0; g < 2; ++g) {
                        cp_scales<CG>(sfa + 4 * g, sfs + g * 32);
                        cp_scales<CG>(sfb + 4 * g * L::kRB, sfs + (L::kSfA >> 4) + g * L::kRB * 32);
                        if (L::kRB == 2 && n > 128) cp_scales<CG>(sfb + 4 * (g * L::kRB + 1), sfs + (L::kSfA >> 4) + (g * L::kRB + 1) * 32);
                    }
#pragma unroll
                    for (int q = 0; q < 4; ++q)
                        mma_mxf4<CG>(d, a + 2 * q, b + 2 * q, idesc | sf_half((q & 1) * 2), sfa + 4 * (q >> 1), sfb + 4 * L::kRB * (q >> 1),
                                 k > 0 || q > 0);
                    mma_commit<CG>(&empty[s]);
                    if (k == steps - 1) mma_commit<CG>(&acc_full[buf]);
                }
                ready = __all_sync(0xffffffffu, next_full);
                s = s_next;
                if (s == 0) parity ^= 1u;
            }
            buf ^= 1;
            if (buf == 0) acc_parity ^= 1u;
        }
        // everything issued has left the tensor core before TMEM is given back
        if (elect_one()) mma_commit<CG>(drained);
        __syncwarp();
        unsigned long long until = 0;
        drain_wait(drained, 0, until);
    } else if (warp >= kScaleWarp) {
        // Two warps per 128-row block of scales (the weight rows, then the data rows), which take the pieces of
        // 16 bytes a row (K = 512, two stages) in turn, each reading kPieces of its own ahead.  Lane l owns rows
        // l, l + 32, l + 64 and l + 96.
        // tcgen05.cp wants, for each K = 128, [32 lanes][4 rows][4 scales]: word w of the lane's four rows is
        // one 16-byte store, so nothing is transposed and no two lanes meet in a bank.
        constexpr int kPieces = 2;
        const int blk = (warp - kScaleWarp) % (1 + L::kRB);    // 0: weights; 1 + rb: data rows [128 rb, 128 rb + 128)
        const int turn = (warp - kScaleWarp) / (1 + L::kRB);   // this warp's pieces: even or odd ones
        const int pitch = mx_scale_pitch(p.K);
        const int pieces = (steps + 1) / 2;
        const int left = p.K / kMxBlock - (pieces - 1) * 16;   // scales of the last piece; the padding counts as 1
        const uint32_t one = 0x7f7f7f7fu;                      // scale 1: for rows that do not exist
        uint32_t keep[4];
#pragma unroll
        for (int x = 0; x < 4; ++x) keep[x] = 0xffffffffu >> min(31, max(0, 32 - 8 * (left - 4 * x))) & (left > 4 * x ? 0xffffffffu : 0u);
        uint4 ring[kPieces][4];
        bool valid[kPieces];
        const uint8_t *src[4];
        TileStream<NT, CG> stream(p, order, tiles);
        int piece = 0;
        int whose = 0;                                         // turn of the next piece
        auto fetch = [&](uint4 (&v)[4]) {                      // this warp's next piece, over all tiles; false when there is none
            int mine;
            do {
                if (piece == 0) {
                    Tile t;
                    if (!stream.next(t)) return false;
                    t.feat += rank * kFeat;
#pragma unroll
                    for (int g = 0; g < 4; ++g) {
                        const int r = lane + 32 * g + (blk > 0 ? (blk - 1) * 128 : 0);
                        const int f = t.feat + (GATED ? weight_row(r) : r);
                        if (blk == 0) src[g] = f < p.N ? p.w_scales + ((size_t)t.slot * p.N + f) * pitch : nullptr;
                        else src[g] = r < t.rows ? p.a_scales + (size_t)(t.row + r) * pitch : nullptr;
                    }
                }
                mine = whose == turn ? piece : -1;
                whose ^= 1;
                if (++piece == pieces) piece = 0;
            } while (mine < 0);
#pragma unroll
            for (int g = 0; g < 4; ++g)
                v[g] = src[g] ? __ldg(reinterpret_cast<const uint4 *>(src[g]) + mine) : make_uint4(one, one, one, one);
            return true;
        };
        int s = 0, at = 0;                                     // next stage of the ring, piece of the tile
        unsigned parity = 1;
        bool ok = true;
        auto skip = [&]() {                                    // past the other warp's piece
            s += at * 2 + 1 < steps ? 2 : 1;
            if (s >= STAGES) { s -= STAGES; parity ^= 1u; }
            if (++at == pieces) at = 0;
        };
        if (turn == 1) skip();
#pragma unroll
        for (int d = 0; d < kPieces; ++d) valid[d] = fetch(ring[d]);
        while (ok && valid[0]) {
#pragma unroll
            for (int d = 0; d < kPieces; ++d) {
                if (!ok || !valid[d]) { ok = false; break; }
                uint4 (&v)[4] = ring[d];
                if (at == pieces - 1 && left < 16) {
#pragma unroll
                    for (int g = 0; g < 4; ++g)
                        v[g] = make_uint4((v[g].x & keep[0]) | (one & ~keep[0]), (v[g].y & keep[1]) | (one & ~keep[1]),
                                          (v[g].z & keep[2]) | (one & ~keep[2]), (v[g].w & keep[3]) | (one & ~keep[3]));
                }
                // both stages of the piece behind one proxy fence
                const bool two = at * 2 + 1 < steps;
                const int s1 = s + 1 == STAGES ? 0 : s + 1;
                const unsigned parity1 = s1 ? parity : parity ^ 1u;
                ok = wait_for<CG>(&empty[s], parity, quit, p.spin_limit);
                ok = __all_sync(0xffffffffu, ok && (!two || wait_for<CG>(&empty[s1], parity1, quit, p.spin_limit)));
                if (!ok) break;
                const int off = (blk == 0 ? 0 : L::kSfA + (blk - 1) * 512) + lane * 16;
                const int next = blk == 0 ? 512 : L::kRB * 512;
                unsigned char *dst = sf + s * L::kSf + off, *dst1 = sf + s1 * L::kSf + off;
                *reinterpret_cast<uint4 *>(dst) = make_uint4(v[0].x, v[1].x, v[2].x, v[3].x);
                *reinterpret_cast<uint4 *>(dst + next) = make_uint4(v[0].y, v[1].y, v[2].y, v[3].y);
                if (two) {
                    *reinterpret_cast<uint4 *>(dst1) = make_uint4(v[0].z, v[1].z, v[2].z, v[3].z);
                    *reinterpret_cast<uint4 *>(dst1 + next) = make_uint4(v[0].w, v[1].w, v[2].w, v[3].w);
                }
                fence_async_shared();
                __syncwarp();
                if (lane == 0) {
                    mbar_arrive_lead<CG>(&full[s]);
                    if (two) mbar_arrive_lead<CG>(&full[s1]);
                }
                s = s1; parity = parity1;
                if (two) {
                    if (++s == STAGES) { s = 0; parity ^= 1u; }
                }
                if (++at == pieces) at = 0;
                skip();
                valid[d] = fetch(v);
            }
        }
    } else if (warp < kEpiWarps) {
        // epilogue: TMEM lane = feature of the tile, column = row
        const int group = warp >> 2, quarter = warp & 3;
        int buf = 0, epi_turn = 0;
        unsigned acc_parity = 0;
        Tile t;
        for (TileStream<NT, CG> stream(p, order, tiles); stream.next(t);) {
            bool ok = wait_for<CG>(&acc_full[buf], acc_parity, quit, p.spin_limit);
            ok = GATED ? warps_all(group + 1, 128, ok) : warps_all((warp >> 1) + 1, 64, ok);   // they meet at barriers below
            if (!ok) break;
            tc_fence_after();
            const uint32_t acc = tmem + buf * NT + ((uint32_t)(quarter * 32) << 16);
            t.feat += rank * kFeat;
            for (int c0 = group * 32; c0 < t.rows; c0 += 64) {
                uint32_t v[32];
                tmem_ld_fragments(acc + c0, v);
                tmem_wait_ld();
                if (c0 + 64 >= t.rows) {                        // this warp's last look at the accumulator
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive_lead<CG>(&acc_empty[buf]);
                }
                unsigned char *epi_buf = epi + (group * L::kEpiBufs + epi_turn) * L::kEpiBuf;   // of the group
                if (GATED) store_gated(p, t, c0, v, reinterpret_cast<float *>(epi_buf), group, quarter, lane);
                else store_plain<L::kEpiBufs>(p, &map_y, t, c0, v, epi_buf + (quarter >> 1) * kBoxBytes, warp >> 1, quarter & 1, lane);
                if (L::kEpiBufs == 2) epi_turn ^= 1;
                else if (GATED) group_sync(group);              // one set of planes: free before the next 32 rows are written
            }
            if (group * 32 >= t.rows && lane == 0) mbar_arrive_lead<CG>(&acc_empty[buf]);
            buf ^= 1;
            if (buf == 0) acc_parity ^= 1u;
        }
        if (!GATED && (quarter & 1) == 0 && lane == 0) bulk_wait_all();   // the last stores have left shared memory
    }

    __syncwarp();
    tc_fence_before();
    if (CG == 2) cluster_sync();                               // the pair leaves together: neither arrives on a CTA that is gone
    else __syncthreads();
    if (*quit) {                                               // in both CTAs of a pair or in none
        // Whichever role gave up, loads may be in flight to this CTA's shared memory: a bounded wait for them (their barriers also
        // count the scales, or are the other CTA's, so they may not complete, but the wait outlasts any copy)
        if (warp == kTmaWarp) {
            unsigned long long until = 0;
            for (int m = max(0, issued - STAGES); m < issued; ++m) drain_wait(&full[m % STAGES], (unsigned)(m / STAGES) & 1u, until);
        }
        __syncwarp();
        if (CG == 2) cluster_sync();
        if (tid == 0) report_status(p.ctl, kDevTimeout);
    }
    if (warp == kMmaWarp) {
        if (CG == 2 && rank == 1) {                            // the first CTA's last arrival is on its way here as well
            unsigned long long until = 0;
            drain_wait(drained, 0, until);
            __syncwarp();
        }
        tc_fence_after();
        tmem_dealloc<CG>(tmem, 512);
    }
}

// ------------------------------------------------------------------------- host

template <int NT, int STAGES, int CG, bool GATED>
cudaError_t launch(const MxProductArgs &a, cudaStream_t st)
{
    using L = Layout<NT, STAGES, CG, GATED>;
    static_assert(L::kEndsOff + 1024 + kMaxP * 4 <= 227 * 1024, "shared memory");
    static_assert(NT >= 32 && NT % 32 == 0, "row boxes and epilogue chunks are 32 rows");
    const auto kernel = k_mx_product<NT, STAGES, CG, GATED>;
    // a function's attributes are those of one device
    constexpr int kDevices = 64;
    static std::once_flag once[kDevices];
    static cudaError_t attr[kDevices];
    if (a.device < 0 || a.device >= kDevices) return cudaErrorInvalidDevice;
    std::call_once(once[a.device], [&] {
        attr[a.device] = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                              (int)std::max(L::bytes(kMaxP), L::bytes(kFullTableP)));
    });
    if (attr[a.device] != cudaSuccess) return attr[a.device];
    if (!encode_fn()) return cudaErrorNotSupported;
    CUtensorMap map_w, map_a, map_big, map_y = {};
    const cuuint64_t row = (cuuint64_t)a.K / 2;
    const cuuint64_t wd[3] = {row, (cuuint64_t)a.N, (cuuint64_t)a.P}, ws[2] = {row, row * (cuuint64_t)a.N};
    const cuuint64_t ad[2] = {row, (cuuint64_t)a.rows}, as[1] = {row};
    const CUtensorMapDataType u8 = CU_TENSOR_MAP_DATA_TYPE_UINT8;
    const CUtensorMapSwizzle sw = CU_TENSOR_MAP_SWIZZLE_128B;
    // the order of weight_row: a row's bytes, the eight rows of one parity, the two parities, the sixteens, the slots
    const cuuint64_t pd[5] = {row, 8, 2, (cuuint64_t)a.N / 16, (cuuint64_t)a.P}, ps[4] = {2 * row, row, 16 * row, row * (cuuint64_t)a.N};
    bool ok = (GATED ? encode(&map_w, u8, sw, a.w_codes, 5, pd, ps, kRowBytes, 8, 2, kFeat / 16)
                     : encode(&map_w, u8, sw, a.w_codes, 3, wd, ws, kRowBytes, kFeat)) &&
              encode(&map_a, u8, sw, a.a_codes, 2, ad, as, kRowBytes, 32) && encode(&map_big, u8, sw, a.a_codes, 2, ad, as, kRowBytes, NT / CG);
    if (!GATED) {
        const cuuint64_t yd[2] = {(cuuint64_t)a.N, (cuuint64_t)a.rows}, ys[1] = {2 * (cuuint64_t)a.N};
        ok = ok && encode(&map_y, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, sw, a.y, 2, yd, ys, 64, 32);
    }
    if (!ok) return cudaErrorInvalidValue;
    KernelParams p;
    p.a_scales = a.a_scales; p.w_scales = a.w_scales; p.slot_counts = a.slot_counts; p.slot_offsets = a.slot_offsets;
    p.rows = a.rows; p.P = a.P; p.N = a.N; p.K = a.K; p.y = static_cast<__nv_bfloat16 *>(a.y);
    p.h_codes = a.h_codes; p.h_scales = a.h_scales; p.ctl = a.ctl; p.spin_limit = a.spin_limit;
    // no more CTAs than there can be tiles (the counts are on the device)
    const long long feats = (a.N + CG * kFeat - 1) / (CG * kFeat);
    const long long most = feats * (std::min<long long>(a.P, a.rows) + a.rows / NT);
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(CG * std::min<long long>(a.sm_count / CG, most)));
    cfg.blockDim = dim3(L::kThreads); cfg.dynamicSmemBytes = L::bytes(a.P); cfg.stream = st;
    cudaLaunchAttribute at[2];
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim.x = CG; at[0].val.clusterDim.y = 1; at[0].val.clusterDim.z = 1;
    at[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = at; cfg.numAttrs = a.pdl ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, kernel, map_w, map_a, map_big, map_y, p);
}

template <bool GATED>
cudaError_t launch_for(const MxProductArgs &a, cudaStream_t st)
{
    // With few rows a slot the weights dominate, and a narrow tile of one CTA leaves shared memory for more
    // stages of them.  With many rows the products do, and a pair of CTAs halves what each holds of the row operand in
    // shared memory (a stage of 256 is written once and read once): 524 clocks a stage, of which the products need 448.
    // Up to 64 rows a slot the two are within 5 % (32 slots of 8 to 64 rows, H 4096, 2048 features: gated 67.6-69.6 us
    // narrow, 67.6-69.7 wide; down 38.9-41.2 and 38.9-41.0).  The host knows the buffer's rows but not the counts, so the
    // mean over all slots, empty ones included, decides.  Where the rows fall on a few slots that costs up to half
    // (n rows on 8 of 288 slots, H 7168, 2048 features, narrow and wide: gated 51.2 and 45.1 us for n = 1024, 125 and 72
    // for 4096, 436 and 182 for 16384; down 32.8 and 28.7, 76 and 43, 256 and 105).
    if (a.rows <= 64ll * a.P) return launch<64, 7, 1, GATED>(a, st);
    return launch<224, 5, 2, GATED>(a, st);
}

}  // namespace

namespace moe {

cudaError_t mx_product_launch(const MxProductArgs &a, cudaStream_t st)
{
    return a.gated ? launch_for<true>(a, st) : launch_for<false>(a, st);
}

}  // namespace moe
