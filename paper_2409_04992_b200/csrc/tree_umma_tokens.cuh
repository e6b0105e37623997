// Attention of draft trees with at most 64 query rows per KV head on the fifth-generation tensor cores, head
// sizes 64, 128 and 256, for sm_100a.  (Work split and copies: tree_umma_common.cuh.)
//
// The TOKENS are the long side of the MMAs, the rows (N = 16, 32 or 64 of them) the short one:
//   S^T[128 tokens x N]  = K_tile[128 x D] Q^T[D x N]
//   O^T[128 dims x 2 N] += V_tile^T[128 x 128] P^T[128 x 2 N]     (head size 256: two accumulators; 64: the
//                                                                  dims twice, the upper half is not read)
// so that exponentials and MMAs are paid for the rows that there are: at 64 rows half of what the form
// with the rows as the long side takes (there a tile costs 128 exponentials a thread whatever the rows
// are, and the MMAs' power holds the clock at 1.45 GHz).  From 32 rows on two groups of four softmax warps
// take half of the rows each, so that a scheduler has two warps whose waits and exponentials overlap.  Thread
// t of a group owns token t: it reads its logits, masks them, and writes its weights to shared memory, each as an
// fp16 high and low part (2 N columns, added up at the end; see tree_umma_rows.cuh for why, and one MMA for both
// because with so few columns the MMA's time is that of reading the V tile).  The rows' references are alike in all
// threads of a group and follow the maximum lazily: a vote per tile says whether any logit exceeds its row's
// by more than kGroupLag, and only then maxima are exchanged and the accumulator rescaled.  A thread keeps
// its own share of the rows' sums.
//
// Measured (K and V bytes per second, 16 sequences of 4k to 8k tokens, 40 KV heads, head size 128, 32-token blocks,
// with the merge; short runs of ten calls, sustained ones in brackets): 8 rows 6.3 TB/s (6.3), 16 rows 6.2 (6.2), 32
// rows 6.0 (5.8; memory is the bound), 64 rows 5.5 (4.9), where the exponentials and the MMAs' power (the clock falls to
// 1.5 GHz) weigh as much as memory.  Head size 256, 20 heads: 16 rows 6.3 (6.2), 64 rows 5.7 (5.2).
#pragma once

#include "tree_umma_common.cuh"

namespace instinfer {

template <int D, int N>
struct TreeTokensGeometry {
    static_assert(N == 16 || N == 32 || N == 64, "row counts of the instances");
    static constexpr int kQPanel = N * 128;                              // 64 dims of N rows
    static constexpr int kQBytes = D / 64 * kQPanel;
    static constexpr int kPBytes = 2 * N * kTreeTile * 2;                // high and low parts
    static constexpr int kGroups = N == 16 ? 1 : 2;                      // of four softmax warps
    static constexpr int kCols = N / kGroups;                            // rows of a group
    static constexpr int kThreads = (4 * kGroups + 4) * 32;
    static constexpr int kExtraBytes = kTreeMiscBytes + N * 20;          // row maxima or sums by warp, and references
    using Ring = TreeRing<D, 226 * 1024 - kQBytes - kPBytes - kExtraBytes>;
    static constexpr int kQOffset = Ring::kRingBytes;
    static constexpr int kPOffset = kQOffset + kQBytes;
    static constexpr int kMiscOffset = kPOffset + kPBytes;
    static constexpr int kSmemBytes = kMiscOffset + kExtraBytes + 1024;  // room to align to 1024 bytes
    static constexpr int kAccs = D == 256 ? 2 : 1;
    static constexpr int kOColumn = 2 * N;                               // tensor memory: two logit buffers, then the accumulators
    static constexpr int kTmemCols = (kOColumn + kAccs * 2 * N > 256) ? 512 : (kOColumn + kAccs * 2 * N > 128) ? 256 :
                                     (kOColumn + kAccs * 2 * N > 64) ? 128 : 64;
    static_assert(kOColumn + kAccs * 2 * N <= kTmemCols, "tensor memory");
    static_assert(kSmemBytes <= 227 * 1024, "one block per SM must fit");
};

// Barriers of one group of 128 softmax threads: `id` 1 (or 3) with a vote, 2 (or 4) without.
__device__ __forceinline__ bool group_any(int id, bool mine)
{
    unsigned out;
    asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.b32 q, %1, 0;\n\tbar.red.or.pred p, %2, 128, q;\n\t"
                 "selp.u32 %0, 1, 0, p;\n\t}" : "=r"(out) : "r"((unsigned)mine), "r"(id) : "memory");
    return out != 0;
}
__device__ __forceinline__ void group_sync(int id) { asm volatile("bar.sync %0, 128;" :: "r"(id) : "memory"); }

// 16 columns of tensor memory; valid after tc_loaded16.
__device__ __forceinline__ void tc_issue_load16(float *v, unsigned taddr)
{
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 "
                 "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
                 : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]), "=f"(v[4]), "=f"(v[5]), "=f"(v[6]), "=f"(v[7]),
                   "=f"(v[8]), "=f"(v[9]), "=f"(v[10]), "=f"(v[11]), "=f"(v[12]), "=f"(v[13]), "=f"(v[14]), "=f"(v[15])
                 : "r"(taddr) : "memory");
}
__device__ __forceinline__ void tc_loaded16(float *v)
{
    asm volatile("tcgen05.wait::ld.sync.aligned;"
                 : "+f"(v[0]), "+f"(v[1]), "+f"(v[2]), "+f"(v[3]), "+f"(v[4]), "+f"(v[5]), "+f"(v[6]), "+f"(v[7]),
                   "+f"(v[8]), "+f"(v[9]), "+f"(v[10]), "+f"(v[11]), "+f"(v[12]), "+f"(v[13]), "+f"(v[14]), "+f"(v[15])
                 :: "memory");
}

template <int D, bool kPaged, int N>
__global__ void __launch_bounds__(TreeTokensGeometry<D, N>::kThreads, 1)
tree_attn_tokens_kernel(const __grid_constant__ TreeParams p, const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_k,
                        const __grid_constant__ CUtensorMap map_v)
{
    using Geo = TreeTokensGeometry<D, N>;
    using Ring = typename Geo::Ring;
    constexpr int kItems = Ring::kItems, kItemPanels = Ring::kItemPanels, kItemBytes = Ring::kItemBytes;
    constexpr int kKSlots = Ring::kKSlots, kVSlots = Ring::kVSlots, kAccs = Geo::kAccs;
    constexpr int kSoftmaxWarps = 4 * Geo::kGroups, kCols = Geo::kCols;
    constexpr int kWarpK = kSoftmaxWarps, kWarpV = kWarpK + 1, kWarpLogits = kWarpK + 2, kWarpOutput = kWarpK + 3;
    extern __shared__ unsigned char smem_raw[];
    const AttnParams &a = p.a;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    allow_next_kernel();
    wait_for_previous_kernels();

    const unsigned raw = static_cast<unsigned>(__cvta_generic_to_shared(smem_raw));
    const unsigned base = (raw + 1023u) & ~1023u;
    unsigned char *smem = smem_raw + (base - raw);
    const unsigned q_smem = base + Geo::kQOffset, p_smem = base + Geo::kPOffset, misc = base + Geo::kMiscOffset;
    unsigned char *misc_ptr = smem + Geo::kMiscOffset;

    tree_count_tiles(p, misc_ptr, Geo::kThreads);
    if (warp == kWarpLogits) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;"
                     :: "r"(misc + kTreeTmemPtr), "n"(Geo::kTmemCols) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    } else if (warp == kWarpK) {
        if (lane == 0) tree_init_barriers(misc, misc_ptr, kSoftmaxWarps, kSoftmaxWarps);
    } else if (warp < kSoftmaxWarps) {
        // rows that do not exist are zeros for good: the copies fill only the others
        const uint4 zero = make_uint4(0u, 0u, 0u, 0u);
        for (int i = threadIdx.x; i < Geo::kQBytes / 16; i += kSoftmaxWarps * 32) *reinterpret_cast<uint4 *>(smem + Geo::kQOffset + i * 16) = zero;
        fence_async_proxy();
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const unsigned tmem = *reinterpret_cast<volatile unsigned *>(misc_ptr + kTreeTmemPtr);
    const TreeQueue queue{misc, misc_ptr};
    const TreeCopies<D, kPaged, Ring> copies{p, smem, base, misc, lane};

    if (warp == kWarpK) {
        copies.template produce_k<1, Geo::kQPanel>(queue, &map_q, &map_k, q_smem);
    } else if (warp == kWarpV) {
        copies.produce_v(queue, &map_v);
    } else if (warp == kWarpLogits) {
        // ================================ logit MMAs ================================
        constexpr unsigned idesc = umma_idesc(128, N, 0, 0);           // K tile and query rows K-major
        const uint64_t q_desc = umma_desc(q_smem, 16, 1024, 2);
        bool fine = true;
        int g = 0;
        for (int k = 0; fine; ++k) {
            fine = queue.wait(k);
            if (!fine) break;
            const TreeSegment seg = queue.entry(k);
            queue.done(k, lane);
            if (seg.b < 0) break;
            fine = __all_sync(0xffffffffu, tree_wait(misc + kTreeBarQFull, k & 1));
            for (int j = seg.t0; j < seg.t1 && fine; ++j, ++g) {
                const int buf = g & 1;
                if (g >= 2) fine = __all_sync(0xffffffffu, tree_wait(misc + kTreeBarSFree + buf * 8, ((g >> 1) - 1) & 1));
#pragma unroll
                for (int item = 0; item < kItems; ++item) {
                    if (!fine) break;
                    const int n = g * kItems + item, slot = n % kKSlots;
                    fine = __all_sync(0xffffffffu, tree_wait(misc + kTreeBarKFull + slot * 8, (n / kKSlots) & 1));
                    if (!fine) break;
                    tc_fence_after();
                    // rows of 128 bytes per 64-dim panel, 8-row groups 1024 bytes apart; a k-step of 16
                    // dims is 32 bytes along the row
                    const uint64_t k_desc = umma_desc(base + slot * kItemBytes, 16, 1024, 2);
                    if (elect_one()) {
#pragma unroll
                        for (int ks = 0; ks < 4 * kItemPanels; ++ks)
                            tc_mma_f16(tmem + buf * N, k_desc + (uint64_t)(((ks >> 2) * kTreePanelBytes + (ks & 3) * 32) >> 4),
                                       q_desc + (uint64_t)(((item * kItemPanels + (ks >> 2)) * Geo::kQPanel + (ks & 3) * 32) >> 4), idesc,
                                       item > 0 || ks > 0);
                        tc_commit(misc + kTreeBarKEmpty + slot * 8);
                        if (item + 1 == kItems) {
                            tc_commit(misc + kTreeBarSFull + buf * 8);
                            if (j + 1 == seg.t1) tc_commit(misc + kTreeBarQEmpty);
                        }
                    }
                    __syncwarp();
                }
            }
        }
        if (!fine && lane == 0 && a.status) atomicOr(a.status, kFlagCopyTimeout);
    } else if (warp == kWarpOutput) {
        // ================================ output MMAs ================================
        constexpr unsigned idesc = umma_idesc(128, 2 * N, 1, 1);       // V tile and weights MN-major
        // Weights: 8-column blocks of [128 tokens][16 bytes], 2048 bytes apart; 8-token groups 128 bytes
        // apart; a k-step is 16 tokens = 256 bytes.  The low parts lie behind the high ones.
        const uint64_t p_desc = umma_desc(p_smem, 128, 2048, 0);
        bool fine = true;
        int g = 0;
        for (int k = 0; fine; ++k) {
            fine = queue.wait(k);
            if (!fine) break;
            const TreeSegment seg = queue.entry(k);
            queue.done(k, lane);
            if (seg.b < 0) break;
            for (int j = seg.t0; j < seg.t1 && fine; ++j, ++g) {
                fine = __all_sync(0xffffffffu, tree_wait(misc + kTreeBarPFull, g & 1));
#pragma unroll
                for (int item = 0; item < kItems; ++item) {
                    if (!fine) break;
                    const int n = g * kItems + item, slot = n % kVSlots;
                    fine = __all_sync(0xffffffffu, tree_wait(misc + kTreeBarVFull + slot * 8, (n / kVSlots) & 1));
                    if (!fine) break;
                    tc_fence_after();
                    // V item read MN-major (M = 128 dims): its 64-dim panels kTreePanelBytes apart (the same panel
                    // twice at head size 64), 8-token groups 1024 bytes apart; a k-step is 16 tokens = 2048 bytes
                    const uint64_t v_desc = umma_desc(base + Ring::kVOffset + slot * kItemBytes, D == 64 ? 0 : kTreePanelBytes, 1024, 2);
                    if (elect_one()) {
                        const unsigned acc = tmem + Geo::kOColumn + item * 2 * N;
#pragma unroll
                        for (int ks = 0; ks < 8; ++ks)
                            tc_mma_f16(acc, v_desc + (uint64_t)((ks * 2048) >> 4), p_desc + (uint64_t)((ks * 256) >> 4), idesc,
                                       j > seg.t0 || ks > 0);
                        tc_commit(misc + kTreeBarVEmpty + slot * 8);
                        if (item + 1 == kItems) tc_commit(misc + kTreeBarPvDone);
                    }
                    __syncwarp();
                }
            }
        }
        if (!fine && lane == 0 && a.status) atomicOr(a.status, kFlagCopyTimeout);
    } else {
        // ================================ softmax and epilogue ================================
        const int group = warp >> 2;                                  // this warp's rows: [row0, row0 + kCols)
        const int row0 = group * kCols, vote_id = 1 + 2 * group, sync_id = 2 + 2 * group;
        const int t = threadIdx.x & 127;                              // token of the tile = lane of tensor memory
        const unsigned lanes = tmem + ((unsigned)((warp & 3) * 32) << 16);
        float *by_warp = reinterpret_cast<float *>(misc_ptr + kTreeMiscBytes);   // [N][4]: a row's maxima, or sums, by warp
        float *offsets = by_warp + N * 4;                             // [N]: the rows' references (negated) as they were last moved
        const int rows_here = p.nodes_per_block * p.group;            // <= N: all the tree's rows
        const int group_inverse = 65536 / p.group + 1;
        auto node_of = [&](int r) -> int { return r * group_inverse >> 16; };      // r / p.group (exact for r < 64)
        const int q_heads = a.heads * p.group;
        const float scale = a.scale_log2e, sign = copysignf(1.f, scale);
        constexpr float kTooLarge = kGroupLag + kGroupWeightLog2;
        bool fine = true;
        float x[kCols];
        // Waits for the logits of a tile and asks for this thread's.
        auto request = [&](int tile) {
            if (fine) fine = tree_wait(misc + kTreeBarSFull + (tile & 1) * 8, (tile >> 1) & 1);
            fine = __all_sync(0xffffffffu, fine);
            tc_fence_after();
#pragma unroll
            for (int r = 0; r < kCols; r += 16) tc_issue_load16(x + r, lanes + (tile & 1) * N + row0 + r);
        };
        int g = 0;
        for (int k = 0;; ++k) {
            // (one decision for the group: its barriers have to stay in step)
            if (group_any(vote_id, !queue.wait(k) || !fine)) {
                fine = false;
                break;
            }
            const TreeSegment &seg = queue.entry(k);                  // read where it is needed: registers are scarce
            if (seg.b < 0) break;
            const int prefix = seg.prefix(), t0 = seg.t0, t1 = seg.t1;
            unsigned *poison = reinterpret_cast<unsigned *>(misc_ptr + kTreePoison) + (k & 7) * 4;
            // (the words of four segments ahead: no warp is more than two segments from another)
            if (threadIdx.x < 4) reinterpret_cast<volatile unsigned *>(misc_ptr + kTreePoison)[((k + 4) & 7) * 4 + threadIdx.x] = 0u;
            const int live_rows = min(rows_here, seg.nodes * p.group);
            // What the group's rows see of the tree, lane r row row0 + r: asked for here, looked at in the last tiles
            // (by loads that the compiler does not move, nor waits for before they are used).
            const bool my_row = t1 * kTreeTile > prefix && lane < kCols && row0 + lane < live_rows;
            uint64_t my_lo = 0, my_hi = 0;
            if (my_row) {
                const uint64_t *words = p.tree.mask + ((int64_t)seg.b * p.tree.tokens + node_of(row0 + lane)) * p.tree.words;
                asm volatile("ld.global.b64 %0, [%1];" : "=l"(my_lo) : "l"(words) : "memory");
                if (p.tree.words > 1) asm volatile("ld.global.b64 %0, [%1];" : "=l"(my_hi) : "l"(words + 1) : "memory");
            }
            // Two rows at a time: the negated reference, and this thread's sums; sums and accumulator carry
            // kGroupWeightScale.  The reference is a logit before it is scaled, taken off before the scale comes in:
            // the largest logit's weight is exactly kGroupWeightScale then, however large it is.
            float2 offset[kCols / 2], l[kCols / 2];
#pragma unroll
            for (int r = 0; r < kCols / 2; ++r) {
                offset[r] = make_float2(-kMinusHuge * sign, -kMinusHuge * sign);
                l[r] = make_float2(0.f, 0.f);
            }
            for (int j = t0; j < t1; ++j, ++g) {
                const int buf = g & 1, start = j * kTreeTile;
                const unsigned logits = lanes + buf * N + row0;
                const bool masked = start + kTreeTile > prefix;       // uniform
                unsigned seen_by = ~0u;                               // the group's rows that see this thread's token
                if (masked) {
                    // The 32 tokens of this warp are columns of the rows' bits: 32 votes transpose them.
                    const int first = start + (warp & 3) * 32 - prefix;            // the node of lane 0's token
                    const TreeRow mine = TreeRow{my_lo, my_hi, my_row}.cut(seg.nodes);
                    const Bits128 bits = {mine.lo, mine.hi};
                    unsigned window = my_row ? ~0u : 0u;
                    if (first >= 0) window = first < 128 ? bits.shifted_down(first).word(0) : 0u;
                    else if (first > -32) window = bits.word(0) << -first | (my_row ? (1u << -first) - 1u : 0u);
#pragma unroll 8
                    for (int i = 0; i < 32; ++i) {
                        const unsigned rows = __ballot_sync(0xffffffffu, window >> i & 1u);
                        if (lane == i) seen_by = rows;
                    }
                }
                request(g);
                // Exponents of the weights against the references; where one is too large the references move
                // and they are computed again.
                float e[kCols];
                for (int attempt = 0;; ++attempt) {
#pragma unroll
                    for (int r = 0; r < kCols; r += 16) tc_loaded16(x + r);
                    float most = -INFINITY, most_odd = -INFINITY;
#pragma unroll
                    for (int r = 0; r < kCols / 2; ++r) {
                        const float2 y = fma2(add2(make_float2(x[2 * r], x[2 * r + 1]), offset[r]), make_float2(scale, scale),
                                              make_float2(kGroupWeightLog2, kGroupWeightLog2));
                        e[2 * r] = y.x;
                        e[2 * r + 1] = y.y;
                    }
                    if (masked) {
#pragma unroll
                        for (int r = 0; r < kCols; ++r)
                            if (!(seen_by >> r & 1u)) e[r] = -INFINITY;
                    }
#pragma unroll
                    for (int r = 0; r < kCols; r += 4) {
                        most = max3(most, e[r], e[r + 1]);
                        most_odd = max3(most_odd, e[r + 2], e[r + 3]);
                    }
                    if (attempt > 0 || !group_any(vote_id, fmaxf(most, most_odd) > kTooLarge)) break;
                    // ---- some row's reference moves (rare after a segment's first tile) ----
                    if (j > t0) {                                 // the accumulator holds the tiles before this one
                        if (fine) fine = tree_wait(misc + kTreeBarPvDone, (g - 1) & 1);
                        fine = __all_sync(0xffffffffu, fine);
                        tc_fence_after();
                    }
#pragma unroll
                    for (int r0 = 0; r0 < kCols; r0 += 16) {
                        float z[16];
                        tc_issue_load16(z, logits + r0);
                        tc_loaded16(z);
#pragma unroll
                        for (int r = 0; r < 16; ++r) z[r] = seen_by >> (r0 + r) & 1u ? z[r] * sign : -INFINITY;
                        const float top = warp_reduce16<true>(z, lane);
                        if ((lane & 1) == 0) by_warp[(row0 + r0 + warp_reduce16_row(lane)) * 4 + (warp & 3)] = top;
                    }
                    group_sync(sync_id);
#pragma unroll
                    for (int r0 = 0; r0 < kCols; r0 += 16) {
                        float alpha[16];
#pragma unroll
                        for (int r = 0; r < 16; ++r) {
                            const float4 tops = *reinterpret_cast<const float4 *>(by_warp + (row0 + r0 + r) * 4);
                            const float top = max3(fmaxf(tops.x, tops.y), tops.z, tops.w);
                            float &off = (r & 1) ? offset[(r0 + r) / 2].y : offset[(r0 + r) / 2].x;
                            float &sum = (r & 1) ? l[(r0 + r) / 2].y : l[(r0 + r) / 2].x;
                            alpha[r] = 1.f;
                            const float moved = -top * sign, rise = (off - moved) * scale;
                            if (rise > kGroupLag) {
                                alpha[r] = fast_exp2(-rise);                              // 2^(old - new reference)
                                off = moved;
                                if (t == r0 + r) offsets[row0 + r0 + r] = off;
                            }
                            sum *= alpha[r];
                        }
                        if (j > t0) {
#pragma unroll
                            for (int part = 0; part < 2 * kAccs; ++part) {        // high and low parts of each accumulator
                                float o[16];
                                tc_issue_load16(o, lanes + Geo::kOColumn + part * N + row0 + r0);
                                tc_loaded16(o);
#pragma unroll
                                for (int r = 0; r < 16; ++r) o[r] *= alpha[r];
                                tc_store16(lanes + Geo::kOColumn + part * N + row0 + r0, o);
                            }
                        }
                    }
                    group_sync(sync_id);                              // the maxima have been read
#pragma unroll
                    for (int r = 0; r < kCols; r += 16) tc_issue_load16(x + r, logits + r);
                }
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbarrier_arrive(misc + kTreeBarSFree + buf * 8);
                unsigned hi[kCols / 2], lo[kCols / 2];
#pragma unroll
                for (int r = 0; r < kCols / 2; ++r) {
                    const float2 w = make_float2(fast_exp2(e[2 * r]), fast_exp2(e[2 * r + 1]));
                    l[r] = add2(l[r], w);
                    hi[r] = pack_half2(w.x, w.y);
                    const float2 back = __half22float2(*reinterpret_cast<const __half2 *>(&hi[r]));
                    const float2 rest = fma2(back, make_float2(-1.f, -1.f), w);
                    lo[r] = pack_half2(rest.x, rest.y);
                }
                if (g > 0) {                                          // the previous tile's MMAs have read the weights
                    if (fine) fine = tree_wait(misc + kTreeBarPvDone, (g - 1) & 1);
                }
                // (late, so that the value tile has had time to land)
                if (masked) copies.template clean_values<32 / Geo::kGroups>(seg, j, g, (warp & 3) * 32 + group * (32 / Geo::kGroups), poison, fine);
                unsigned char *weights = smem + Geo::kPOffset + row0 * 256 + t * 16;
#pragma unroll
                for (int r = 0; r < kCols / 2; r += 4) {
                    *reinterpret_cast<uint4 *>(weights + r * 512) = make_uint4(hi[r], hi[r + 1], hi[r + 2], hi[r + 3]);
                    *reinterpret_cast<uint4 *>(weights + N * 256 + r * 512) = make_uint4(lo[r], lo[r + 1], lo[r + 2], lo[r + 3]);
                }
                fence_async_proxy();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbarrier_arrive(misc + kTreeBarPFull);
            }
            // ---- the segment's end: row sums, then the accumulator divided by them; thread t has dim t ----
#pragma unroll
            for (int r0 = 0; r0 < kCols; r0 += 16) {
                float x[16];
#pragma unroll
                for (int r = 0; r < 16; ++r) x[r] = (r & 1) ? l[(r0 + r) / 2].y : l[(r0 + r) / 2].x;
                const float sum = warp_reduce16<false>(x, lane);
                if ((lane & 1) == 0) by_warp[(row0 + r0 + warp_reduce16_row(lane)) * 4 + (warp & 3)] = sum;
            }
            group_sync(sync_id);
            const bool whole = seg.whole();
            if (t < kCols) {
                // one thread per row: its sum's inverse (0: a row of zeros) and its log-sum-exp
                const int r = row0 + t;
                const float4 sums = *reinterpret_cast<const float4 *>(by_warp + r * 4);
                const float total = (sums.x + sums.y) + (sums.z + sums.w);
                const bool empty = r >= live_rows || total == 0.f;    // (a NaN sum is not an empty row's)
                const float lse2 = empty ? kMinusHuge : log2f(total) - fmaf(offsets[r], scale, kGroupWeightLog2);
                if (r < rows_here && fine) {
                    const int node = node_of(r);
                    if (!whole) seg.lse[r] = lse2;
                    else if (seg.lse) seg.lse[node * q_heads + (r - node * p.group)] = empty ? -INFINITY : lse2 * kLn2;
                }
                *reinterpret_cast<float2 *>(by_warp + r * 4) = make_float2(empty ? 0.f : __fdividef(1.f, total), lse2);
            }
            if (fine) fine = tree_wait(misc + kTreeBarPvDone, (g - 1) & 1);
            fine = __all_sync(0xffffffffu, fine);
            tc_fence_after();
            group_sync(sync_id);
            const volatile unsigned *taken = poison;
            const bool stray = (taken[0] | taken[1] | taken[2] | taken[3]) != 0u;
#pragma unroll 1
            for (int block = 0; block < kCols / 16 * kAccs; ++block) {
                const int first = row0 + block / kAccs * 16, acc = block % kAccs, d = acc * 128 + t;
                float o[16], low[16];
                tc_issue_load16(o, lanes + Geo::kOColumn + acc * 2 * N + first);
                tc_issue_load16(low, lanes + Geo::kOColumn + (acc * 2 + 1) * N + first);
                tc_loaded16(o);
                tc_loaded16(low);
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const float inverse = by_warp[(first + i) * 4];
                    o[i] = inverse == 0.f ? 0.f : (o[i] + low[i]) * inverse;      // (an empty row's accumulator may hold anything)
                }
                const bool writes = fine && (D >= 128 || t < D);
                if (stray) {
                    float more[16];
#pragma unroll 1
                    for (int i = 0; i < 16; ++i)
                        more[i] = writes && first + i < rows_here ? tree_poisoned_value(p, seg, poison, first + i, D, d, by_warp[(first + i) * 4 + 1]) : 0.f;
#pragma unroll
                    for (int i = 0; i < 16; ++i) o[i] += more[i];
                }
                const int rows = writes ? rows_here - first : 0;
                if (whole) {
                    __half *out = static_cast<__half *>(seg.out) + d;
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        const int node = node_of(first + i);
                        if (i < rows) out[(node * q_heads + (first + i - node * p.group)) * D] = __float2half_rn(o[i]);
                    }
                } else {
                    float *out = static_cast<float *>(seg.out) + first * D + d;
#pragma unroll
                    for (int i = 0; i < 16; ++i)
                        if (i < rows) out[i * D] = o[i];
                }
                __syncwarp();
            }
            tc_fence_before();                                        // the accumulator has been read: the next tile may overwrite it
            group_sync(sync_id);                                      // so have the rows' numbers
            queue.done(k, lane);
        }
        if (!fine && lane == 0 && a.status) atomicOr(a.status, kFlagCopyTimeout);
    }

    // ---- teardown: everyone is done with tensor memory before it is released ----
    tc_fence_before();
    __syncthreads();
    if (warp == kWarpLogits) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" :: "r"(tmem), "n"(Geo::kTmemCols) : "memory");
    }
}

}  // namespace instinfer
