// Gradients of the routed step.
//
// combine:   y[t] = sum_j w[t,j] * scale[slot] * buf[row(t,j)]
//   d_buf[row(t,j)] = bf16(w[t,j] * scale[slot] * dy[t])     (the coefficient is one fp32 multiply, as forward)
//   d_w[t,j]        = scale[slot] * <buf[row(t,j)], dy[t]>    (fp32 sums)
// dispatch:  send[row(t,j)] = x[t];  w[t,:] from the logits of the chosen experts
//   d_x[t]          = bf16(sum_j d_send[row(t,j)])            (fp32, ascending j)
//   w_j = c * u_j / sum_i u_i with u = exp(l) or u = sigmoid(l), c = route_scale:
//   d_l_j           = w_j * (g_j - sum_i w_i g_i / c) * (1 for softmax, 1 - sigmoid(l_j) = sigmoid(-l_j) for sigmoid)
//   and zero for every expert that was not chosen (the selection itself has no gradient).
//   Where -inf logits leave a token fewer than k selectable experts, routing fills its last picks with some expert
//   and the constant u = 1 (for softmax u = exp(l - l_0), l_0 the best pick's logit, so 1 is the best pick's own
//   score).  Filled picks take part in the sums and get no gradient; for softmax the selected picks then move
//   against l_0 alone: d_l_0 = - (sum of the other selected picks' d_l), which is the formula above where nothing
//   was filled.
#pragma once

#include "combine_kernels.cuh"

namespace moe {

struct BackwardParams {
    const uint4 *rows;           // [T*k, H/8] combine: the expert rows; dispatch: d_send_buf
    const uint4 *dy;             // [T, H/8]   combine only
    uint4 *out;                  // combine: d_expert_buf [T*k, H/8]; dispatch: dx [T, H/8]
    float *d_weights;            // [T,k] combine: out; dispatch: in (NULL = no gradient of the gate)
    int T, k, hv, P;
    const int32_t *dst_row;      // [T*k]
    const float *topk_weights;   // [T,k]
    const int32_t *topk_slot;    // [T,k]
    const float *slot_scale;     // [P]        combine only
    // gate (dispatch only)
    const int32_t *topk_ids;     // [T,k]
    const float *logits;         // [T,E]; NULL (softmax only) = no token ran out of experts
    float *d_logits;             // [T,E]
    int E, sigmoid;
    int topk_group, group_size;  // group-limited selection; topk_group 0 = none
    float inv_scale;             // 1 / route_scale
    const uint4 *zero_row;       // [H/8] zeros: stands in for a row that was not placed
    Control *ctl;
    unsigned spin_limit;
    int slots;                   // ring slots
    int slot_units;              // 16-byte units per slot
};

constexpr int kBwdWarps = 8;                               // warps that work on the rows; one more copies them
constexpr int backward_threads(bool combine) { return (kBwdWarps + (combine ? 1 : 2)) * 32; }   // ... and one has the gate
constexpr int kBwdUnits = 4;                               // 16-byte units of a slot per thread
constexpr int kBwdSlotUnits = kBwdWarps * 32 * kBwdUnits;  // 16 KB
constexpr int kBwdMaxSlots = 15;
constexpr int kMaxTopKDevice = 16;

// Dynamic tokens without a counter in memory: the grid has a CTA per token, and a resident CTA takes over the
// next one that has not been launched yet (cluster launch control).  The answer arrives in shared memory behind
// an mbarrier, so it is asked for a token ahead.
__device__ __forceinline__ void clc_request(void *answer, uint64_t *bar)
{
    mbar_expect_tx(bar, 16);
    asm volatile("clusterlaunchcontrol.try_cancel.async.shared::cta.mbarrier::complete_tx::bytes.b128 [%0], [%1];" ::"r"(smem_addr(answer)),
                 "r"(smem_addr(bar))
                 : "memory");
}

// blockIdx.x of the CTA that was taken over, -1 if none was left (then nothing may be asked again)
__device__ __forceinline__ int clc_answer(const void *answer)
{
    int ok, x;
    asm volatile(
        "{\n\t.reg .b128 r;\n\t.reg .pred p;\n\t"
        "ld.shared.b128 r, [%2];\n\t"
        "clusterlaunchcontrol.query_cancel.is_canceled.pred.b128 p, r;\n\t"
        "selp.s32 %0, 1, 0, p;\n\tmov.s32 %1, 0;\n\t"
        "@p clusterlaunchcontrol.query_cancel.get_first_ctaid::x.b32.b128 %1, r;\n\t}"
        : "=r"(ok), "=r"(x)
        : "r"(smem_addr(answer))
        : "memory");
    return ok ? x : -1;
}

struct BackwardTable {                                     // one token's assignments
    int token;                                             // -1: no more
    int row[kMaxTopKDevice];
    float coef[kMaxTopKDevice], scale[kMaxTopKDevice];
};

inline size_t backward_smem(int slots, int slot_units) { return (size_t)slots * slot_units * 16 + 128; }

// Gradient of the gate for one token, by one warp: lanes j < k form the k values, the row of d_logits is cleared
// and the values written into it (__syncwarp orders the two).
//
// Which picks were filled follows from what was picked.  Selected picks come first, are distinct and not masked.
// Filled ones all name one expert that has a live replica.  If that expert is masked, its logit says so.  If not,
// it either was selected before (so the pick repeats an earlier one), or its group was not kept; then every kept
// group had a selectable expert and, as routing ran out, all of those were picked: the earlier picks lie in
// topk_group groups and this one in yet another.  No selected pick has any of the three marks.
__device__ __forceinline__ void route_backward(const BackwardParams &p, int t, int lane)
{
    const unsigned full = 0xffffffffu;
    float w = 0.0f, g = 0.0f, slope = 1.0f;
    int id = -1;
    bool filled = false;
    if (lane < p.k) {
        const size_t i = (size_t)t * p.k + lane;
        id = __ldg(p.topk_ids + i);
        w = __ldg(p.topk_weights + i);
        g = __ldg(p.d_weights + i);
        if ((unsigned)id >= (unsigned)p.E) id = -1;
    }
    // A filled last pick has the largest score there is: unless no pick weighs more than the last one, there is
    // nothing to look for (and with softmax no need to fetch logits behind the ids).
    const float w_last = __shfl_sync(full, w, p.k - 1);
    const bool look = __all_sync(full, lane >= p.k || w <= w_last);
    if ((look || p.sigmoid) && lane < p.k) {
        filled = id < 0;
        if (p.logits && id >= 0) {
            const float l = __ldg(p.logits + (size_t)t * p.E + id);
            filled = l == __int_as_float(0xff800000);
            if (p.sigmoid) slope = sigmoid_spec(-l);           // 1 - sigmoid(l) without cancellation
        }
    }
    // g_j - sum_i p_i g_i as sum_i p_i (g_j - g_i) (the p_i = w_i / route_scale add up to 1): nothing
    // cancels where one expert has nearly all of the weight
    float diff = 0.0f;
    for (int i = 0; i < p.k; ++i) {
        const float wi = __shfl_sync(full, w, i), gi = __shfl_sync(full, g, i);
        diff += wi * p.inv_scale * (g - gi);
    }
    float d = w * diff * slope;
    int selected = p.k;
    if (look) {
        filled |= (__match_any_sync(full, id) & lanemask_lt()) != 0u;
        if (p.topk_group) {
            const bool new_group = (__match_any_sync(full, id / p.group_size) & lanemask_lt()) == 0u;
            const unsigned firsts = __ballot_sync(full, new_group && lane < p.k);
            filled |= new_group && __popc(firsts & lanemask_lt()) >= p.topk_group;
        }
        const unsigned marks = __ballot_sync(full, filled && lane < p.k);
        if (marks) {
            selected = __ffs(marks) - 1;
            float others = 0.0f;
            for (int i = 1; i < selected; ++i) others += __shfl_sync(full, d, i);
            if (lane == 0 && !p.sigmoid) d = 0.0f - others;
        }
    }
    float *row = p.d_logits + (size_t)t * p.E;
    if ((p.E & 3) == 0) {
        for (int e = lane * 4; e < p.E; e += 128) *reinterpret_cast<float4 *>(row + e) = make_float4(0.f, 0.f, 0.f, 0.f);
    } else {
        for (int e = lane; e < p.E; e += 32) row[e] = 0.0f;
    }
    __syncwarp();
    if (lane < selected && id >= 0) row[id] = d;
}

// Both gradients: a CTA per token, and as many tokens per CTA as it gets done.  One warp asks the TMA engine for
// the token's rows (dy and the k expert rows; the k rows of d_send_buf), 16 KB of each at a time, through a ring of
// shared-memory slots that runs ahead over tokens.  Eight
// warps take the rows from their slots: for combine they keep the dy row in registers, take each expert row for
// its dot product and write the d_buf row in its place; for dispatch they add the rows up.  Bound by HBM:
// (1 + 2k) rows of traffic per token, or k + 1.  The ring keeps some 200 KB per SM in flight and has the next
// token's rows coming while the present one ends.  Tokens are taken as CTAs get free, because SMs do not get
// equal shares of HBM: dealt out in advance, the SMs were busy for 83 % of the kernel (combine, 8192 tokens of
// 7168, k = 8: 350 us; 304 us like this, 6.56 TB/s).
// Short rows are another matter: a slot holds one piece of one row whatever its length, one lane asks for the rows one
// after the other, and at H = 512 at most 15 KB per CTA are in flight (share of the bytes' time at 300 MB of rows,
// combine and dispatch: H = 512 k = 8 0.22 and 0.12, 1024 0.42 and 0.22, 2048 0.72 and 0.41, 4096 0.91 and 0.70).
// Dot products are summed per thread, over the warp and over the warps, always in the same order.
// K = top_k known at compile time, 0 = any: 8 and 2, the values of the framework's workloads, as in the combine.  The
// variant for any k spills 8 bytes for combine and keeps up (H = 7168, share of the bytes' time: k = 1 0.87, 4 0.91, 6
// 0.89 against 0.93 for 2 and 0.91 for 8).
template <bool COMBINE, int K>
__global__ void __launch_bounds__(backward_threads(COMBINE), 2) k_backward(BackwardParams p)
{
    constexpr int U = kBwdUnits, KK = K > 0 ? K : kMaxTopKDevice;
    extern __shared__ __align__(128) unsigned char ring[];
    __shared__ __align__(8) uint64_t full[kBwdMaxSlots], empty[kBwdMaxSlots];
    __shared__ BackwardTable table[kBwdMaxSlots + 2];
    __shared__ __align__(16) unsigned char clc[16];
    __shared__ __align__(8) uint64_t clc_bar;
    __shared__ float s_dot[2][kBwdWarps][kMaxTopKDevice];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int k = K > 0 ? K : p.k, S = p.slots;
    if (tid == 0) {
        for (int s = 0; s < S; ++s) { mbar_init(&full[s], 1); mbar_init(&empty[s], kBwdWarps + (COMBINE ? 0 : 1)); }
        mbar_init(&clc_bar, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    __syncthreads();
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int chunks = (p.hv + p.slot_units - 1) / p.slot_units;
    const size_t slot_bytes = (size_t)p.slot_units * 16;
    int s = 0;
    bool ok = true;

    if (warp == kBwdWarps) {
        unsigned parity = 1, clc_parity = 0;
        int issued = 0, entry = 0, t = blockIdx.x;
        if (lane == 0) clc_request(clc, &clc_bar);
        int dst; bool placed; float scale, weight;              // lane j < k: assignment j of the token to come
        auto fetch = [&](int tok) {
            dst = -1; placed = false; scale = weight = 0.0f;
            if (tok >= 0 && lane < k) {
                const size_t i = (size_t)tok * k + lane;
                const int slot = __ldg(p.topk_slot + i);
                dst = __ldg(p.dst_row + i);
                placed = (unsigned)slot < (unsigned)p.P && dst >= 0 && dst < (long long)p.T * k;
                if (COMBINE && placed) { scale = __ldg(p.slot_scale + slot); weight = __ldg(p.topk_weights + i); }
            }
        };
        fetch(t);
        while (true) {
            // Table entries are reused after kBwdMaxSlots + 2 tokens; every token takes a slot, and the ring
            // holds no more than kBwdMaxSlots of them besides the one that is being worked on.
            const int row = placed ? dst : -1;                  // lane j < k: row of assignment j
            if (COMBINE && t >= 0 && lane < k) {
                table[entry].row[lane] = row;
                table[entry].scale[lane] = scale;
                table[entry].coef[lane] = placed ? __fmul_rn(weight, scale) : 0.0f;
            }
            if (lane == 0) table[entry].token = t;
            __syncwarp();
            if (t < 0) {                                        // tell the others that there is nothing more
                unsigned spins = 0;
                while (!mbar_try_wait(&empty[s], parity))
                    if (++spins > p.spin_limit) { ok = false; break; }
                if (lane == 0 && ok) asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(smem_addr(&full[s])) : "memory");
                ok = __all_sync(0xffffffffu, ok);
                break;
            }
            for (int c = 0; c < chunks && ok; ++c) {
                const int u0 = c * p.slot_units;
                const unsigned bytes = (unsigned)min(p.slot_units, p.hv - u0) * 16u;
                for (int j = COMBINE ? -1 : 0; j < k; ++j) {    // dy (-1), then the k rows
                    const int r = __shfl_sync(0xffffffffu, row, j < 0 ? 0 : j);
                    unsigned spins = 0;
                    while (!mbar_try_wait(&empty[s], parity))
                        if (++spins > p.spin_limit) { ok = false; break; }
                    ok = __all_sync(0xffffffffu, ok);
                    if (!ok) break;
                    if (lane == 0) {
                        const uint4 *src = j < 0 ? p.dy + (size_t)t * p.hv : r >= 0 ? p.rows + (size_t)r * p.hv : p.zero_row;
                        mbar_expect_tx(&full[s], bytes);        // also publishes the table entry
                        bulk_load(ring + s * slot_bytes, src + u0, bytes, &full[s]);
                    }
                    __syncwarp();
                    ++issued;
                    if (++s == S) { s = 0; parity ^= 1u; }
                }
            }
            if (!ok) break;
            if (++entry == kBwdMaxSlots + 2) entry = 0;
            unsigned spins = 0;
            while (!mbar_try_wait(&clc_bar, clc_parity))
                if (++spins > p.spin_limit) { ok = false; break; }
            ok = __all_sync(0xffffffffu, ok);
            if (!ok) break;
            clc_parity ^= 1u;
            t = clc_answer(clc);
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            __syncwarp();                                       // every lane has read the answer
            if (t >= 0 && lane == 0) clc_request(clc, &clc_bar);
            fetch(t);
        }
        if (!ok) {
            if (lane == 0) report_status(p.ctl, kDevTimeout);
            // the answer and the copies in flight still land in this CTA's shared memory: a bounded wait for each
            unsigned long long until = 0;
            for (int m = max(0, issued - S); m < issued; ++m) drain_wait(&full[m % S], (unsigned)(m / S) & 1u, until);
            drain_wait(&clc_bar, clc_parity, until);           // last: with nothing asked for, this one runs out
        }
        return;
    }

    if (!COMBINE && warp == kBwdWarps + 1) {
        // The gradient of the gate, at its own pace: this warp sees every slot go by (and hands it back at once) and
        // works on a token's gate at its first slot, with a ring's worth of slots before it holds anything up.  From the
        // copying warp it cost 40 of 191 us (8192 tokens, k = 8).
        unsigned parity = 0;
        int entry = 0;
        while (true) {
            for (int m = 0; m < chunks * k && ok; ++m) {
                unsigned spins = 0;
                while (!mbar_try_wait(&full[s], parity))
                    if (++spins > p.spin_limit) { ok = false; break; }
                ok = __all_sync(0xffffffffu, ok);
                const int t = ok ? table[entry].token : -1;
                __syncwarp();
                if (!ok || t < 0) return;
                if (lane == 0) asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(smem_addr(&empty[s])) : "memory");
                if (++s == S) { s = 0; parity ^= 1u; }
                if (m == 0 && p.d_logits) route_backward(p, t, lane);
            }
            if (++entry == kBwdMaxSlots + 2) entry = 0;
        }
    }

    unsigned parity = 0;
    int entry = 0, side = 0;
    auto wait_full = [&]() {
        unsigned spins = 0;
        while (ok && !mbar_try_wait(&full[s], parity))
            if (++spins > p.spin_limit) ok = false;
    };
    auto take = [&](uint4 (&v)[U], int units) {                 // this thread's units of the next slot, which is then handed back
        wait_full();
        const uint4 *src = reinterpret_cast<const uint4 *>(ring + s * slot_bytes);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int c = u * kBwdWarps * 32 + tid;
            v[u] = ok && c < units ? src[c] : make_uint4(0u, 0u, 0u, 0u);
        }
        __syncwarp();
        if (lane == 0) asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(smem_addr(&empty[s])) : "memory");
        if (++s == S) { s = 0; parity ^= 1u; }
    };
    // One barrier a token (the other half of s_dot is used in between), which also makes the warps leave together:
    // a warp that gave up still comes to it.
    auto verdict = [&]() {
        uint32_t good;
        asm volatile("{\n\t.reg .pred a, b;\n\tsetp.ne.u32 a, %1, 0;\n\tbarrier.cta.red.and.pred b, 1, %2, a;\n\tselp.u32 %0, 1, 0, b;\n\t}"
                     : "=r"(good) : "r"((uint32_t)ok), "n"(kBwdWarps * 32) : "memory");
        ok = good != 0;
    };
    while (true) {
        wait_full();                                            // the token's first slot: its table entry is there as well
        const int t = ok ? table[entry].token : 0;
        if (t < 0) { verdict(); break; }
        float dot[KK];
#pragma unroll
        for (int j = 0; j < KK; ++j) dot[j] = 0.0f;
        for (int c = 0; c < chunks; ++c) {
            const int u0 = c * p.slot_units, units = min(p.slot_units, p.hv - u0);
            if constexpr (COMBINE) {
                uint4 g[U];
                take(g, units);
#pragma unroll
                for (int j = 0; j < KK; ++j) {
                    if (K == 0 && j >= k) break;
                    uint4 v[U];
                    take(v, units);
                    const int r = table[entry].row[j];
                    const float coef = table[entry].coef[j];
                    uint4 *dst = p.out + (size_t)max(r, 0) * p.hv + u0;
#pragma unroll
                    for (int u = 0; u < U; ++u) {
                        const int at = u * kBwdWarps * 32 + tid;
                        if (at >= units) break;
                        const __nv_bfloat162 *a = reinterpret_cast<const __nv_bfloat162 *>(&v[u]);
                        const __nv_bfloat162 *b = reinterpret_cast<const __nv_bfloat162 *>(&g[u]);
                        float o[8];
#pragma unroll
                        for (int q = 0; q < 4; ++q) {
                            const float2 fa = __bfloat1622float2(a[q]), fb = __bfloat1622float2(b[q]);
                            dot[j] = __fmaf_rn(fa.x, fb.x, dot[j]);
                            dot[j] = __fmaf_rn(fa.y, fb.y, dot[j]);
                            o[2 * q] = coef * fb.x; o[2 * q + 1] = coef * fb.y;
                        }
                        if (ok && r >= 0) st_stream_v4(dst + at, pack_bf16x8(o));
                    }
                }
            } else {
                float acc[U][8];
#pragma unroll
                for (int u = 0; u < U; ++u)
#pragma unroll
                    for (int q = 0; q < 8; ++q) acc[u][q] = 0.0f;
#pragma unroll
                for (int j = 0; j < KK; ++j) {
                    if (K == 0 && j >= k) break;
                    uint4 v[U];
                    take(v, units);
#pragma unroll
                    for (int u = 0; u < U; ++u) fma_bf16x8(acc[u], v[u], 1.0f);
                }
                uint4 *dst = p.out + (size_t)t * p.hv + u0;
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    const int at = u * kBwdWarps * 32 + tid;
                    if (ok && at < units) st_stream_v4(dst + at, pack_bf16x8(acc[u]));
                }
            }
        }
        if constexpr (COMBINE) {
#pragma unroll
            for (int j = 0; j < KK; ++j) {
                if (K == 0 && j >= k) break;
#pragma unroll
                for (int off = 16; off > 0; off >>= 1) dot[j] += __shfl_xor_sync(0xffffffffu, dot[j], off);
                if (lane == 0) s_dot[side][warp][j] = dot[j];
            }
        }
        verdict();
        if (!ok) break;
        if (COMBINE && tid < k) {
            float sum = 0.0f;
#pragma unroll
            for (int w = 0; w < kBwdWarps; ++w) sum += s_dot[side][w][tid];
            p.d_weights[(size_t)t * k + tid] = table[entry].scale[tid] * sum;
        }
        side ^= 1;
        if (++entry == kBwdMaxSlots + 2) entry = 0;
    }
    if (!ok && tid == 0) report_status(p.ctl, kDevTimeout);
}

}  // namespace moe
