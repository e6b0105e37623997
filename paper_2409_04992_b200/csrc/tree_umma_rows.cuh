// Attention of draft trees with more than 64 query rows per KV head on the fifth-generation tensor cores,
// head sizes 64, 128 and 256, for sm_100a.  (Work split and copies: tree_umma_common.cuh.)
//
// The QUERY ROWS are the long side of the MMAs (fewer rows take tree_umma_tokens.cuh, which has the
// tokens there and pays for the rows that exist):
//   S[128 rows x 128 tokens]  = Q[128 x D] K_tile^T           (both K-major, as they lie in memory)
//   O[128 rows x D]          += P[128 x 128] V_tile           (P from tensor memory, V MN-major)
// A row is a lane of tensor memory and belongs to one thread: its maximum, sum and rescaling need no
// exchange between threads.  The softmax weights go back to tensor memory over the logits they came
// from, each as an fp16 high and low part (P V is then two MMAs): the sum keeps the accuracy of 32-bit
// weights, where one fp16 part alone would add an error as large as the output's own rounding.
//
// kStreams = 1 (at most 128 rows, or head size 256): two logit buffers, so that S of the next tile is
// computed while the softmax warps work on this one.  kStreams = 2: two row blocks share every K and V
// tile; each has its own softmax warps and accumulator, and as tensor memory is full then, its two logit
// buffers hold half a tile each (64 tokens): with one buffer of a whole tile per row block the softmax
// waited for the MMAs that use the weights and for those of the next logits, 2700 of 6100 cycles a tile.
// (Leaving the low parts out in this form gave another 11 % and 1.4 times the error.)
//
// Measured, over 8 x 32k tokens of 8 KV heads, head size 128, the two products counted once (the low parts' MMAs come
// on top): 256 rows (32 nodes x 8 heads) 389 us, 707 TFLOP/s, in short runs and 447 us, 615, sustained; 512 rows 744
// us, 739 TFLOP/s, and 844 us, 651.  Trees of 16 to 32 nodes on the 256 rows 461 us.  The tensor pipe is active 55 % of
// the time, the exponentials' pipe 38 %: what bounds it is the chain logits -> softmax -> weights of a unit, of which a
// block has two (or four half) in flight.  Fewer rows over 16 x 40 heads x 4k to 8k: 80 rows 469 us (542 sustained),
// 128 rows 494 (566); memory alone would take 316.
#pragma once

#include "tree_umma_common.cuh"

namespace instinfer {

template <int D, int kStreams>
struct TreeRowsGeometry {
    static constexpr int kQBytes = D / 64 * kTreePanelBytes;             // per stream
    using Ring = TreeRing<D, 224 * 1024 - kStreams * kQBytes>;
    static constexpr int kQOffset = Ring::kRingBytes;
    static constexpr int kMiscOffset = kQOffset + kStreams * kQBytes;
    static constexpr int kSmemBytes = kMiscOffset + kTreeMiscBytes + 1024;     // room to align to 1024 bytes
    static constexpr int kSoftmaxWarps = 4 * kStreams;
    static constexpr int kThreads = (kSoftmaxWarps + 4) * 32;
    static constexpr int kUnit = kStreams == 1 ? 128 : 64;               // tokens whose logits and weights go through a buffer at once
    static constexpr int kUnits = 128 / kUnit;                           // per tile
    static constexpr int kOColumn = 256;                                 // tensor memory: two logit buffers, then the accumulators
    static_assert(kOColumn + kStreams * D <= 512, "tensor memory");
    static_assert(kSmemBytes <= 227 * 1024, "one block per SM must fit");
};

template <int kWords>
__device__ __forceinline__ void store_row(void *to, const unsigned (&w)[kWords])
{
    if ((reinterpret_cast<uintptr_t>(to) & 31) == 0) {
#pragma unroll
        for (int c = 0; c < kWords; c += 8) {
            const unsigned v[8] = {w[c], w[c + 1], w[c + 2], w[c + 3], w[c + 4], w[c + 5], w[c + 6], w[c + 7]};
            store_32b(static_cast<unsigned char *>(to) + 4 * c, v);
        }
    } else {
#pragma unroll
        for (int c = 0; c < kWords; c += 4)
            *reinterpret_cast<uint4 *>(static_cast<unsigned char *>(to) + 4 * c) = make_uint4(w[c], w[c + 1], w[c + 2], w[c + 3]);
    }
}

template <int D, bool kPaged, int kStreams>
__global__ void __launch_bounds__(TreeRowsGeometry<D, kStreams>::kThreads, 1)
tree_attn_rows_kernel(const __grid_constant__ TreeParams p, const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_k,
                      const __grid_constant__ CUtensorMap map_v)
{
    using Geo = TreeRowsGeometry<D, kStreams>;
    using Ring = typename Geo::Ring;
    constexpr int kItems = Ring::kItems, kItemPanels = Ring::kItemPanels, kItemBytes = Ring::kItemBytes;
    constexpr int kKSlots = Ring::kKSlots, kVSlots = Ring::kVSlots;
    constexpr int kWarpK = Geo::kSoftmaxWarps, kWarpV = kWarpK + 1, kWarpLogits = kWarpK + 2, kWarpOutput = kWarpK + 3;
    extern __shared__ unsigned char smem_raw[];
    const AttnParams &a = p.a;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    allow_next_kernel();
    wait_for_previous_kernels();

    const unsigned raw = static_cast<unsigned>(__cvta_generic_to_shared(smem_raw));
    const unsigned base = (raw + 1023u) & ~1023u;
    unsigned char *smem = smem_raw + (base - raw);
    const unsigned q_smem = base + Geo::kQOffset, misc = base + Geo::kMiscOffset;
    unsigned char *misc_ptr = smem + Geo::kMiscOffset;

    tree_count_tiles(p, misc_ptr, Geo::kThreads);
    if (warp == kWarpLogits) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;"
                     :: "r"(misc + kTreeTmemPtr), "n"(512) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    } else if (warp == kWarpK) {
        if (lane == 0) tree_init_barriers(misc, misc_ptr, 4, Geo::kSoftmaxWarps);
    } else if (warp < Geo::kSoftmaxWarps) {
        // rows of a block that do not exist are zeros for good: the copies fill only the others
        const uint4 zero = make_uint4(0u, 0u, 0u, 0u);
        for (int i = threadIdx.x; i < kStreams * Geo::kQBytes / 16; i += Geo::kSoftmaxWarps * 32)
            *reinterpret_cast<uint4 *>(smem + Geo::kQOffset + i * 16) = zero;
        fence_async_proxy();
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const unsigned tmem = *reinterpret_cast<volatile unsigned *>(misc_ptr + kTreeTmemPtr);
    const TreeQueue queue{misc, misc_ptr};
    const TreeCopies<D, kPaged, Ring> copies{p, smem, base, misc, lane};

    constexpr int kUnit = Geo::kUnit, kUnits = Geo::kUnits;
    // The buffer of a unit (tile number g of this block, stream s, part h of the tile) and how often it was used before.
    auto buffer_of = [](int g, int s, int h) -> int { return kStreams == 1 ? g & 1 : 2 * s + h; };
    auto use_of = [](int g) -> int { return kStreams == 1 ? g >> 1 : g; };

    if (warp == kWarpK) {
        copies.template produce_k<kStreams, kTreePanelBytes>(queue, &map_q, &map_k, q_smem);
    } else if (warp == kWarpV) {
        copies.produce_v(queue, &map_v);
    } else if (warp == kWarpLogits) {
        // ================================ logit MMAs ================================
        constexpr unsigned idesc = umma_idesc(128, kUnit, 0, 0);
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
#pragma unroll
                for (int item = 0; item < kItems; ++item) {
                    if (!fine) break;
                    const int n = g * kItems + item, slot = n % kKSlots;
                    fine = __all_sync(0xffffffffu, tree_wait(misc + kTreeBarKFull + slot * 8, (n / kKSlots) & 1));
                    if (!fine) break;
                    // rows of 128 bytes per 64-dim panel, 8-row groups 1024 bytes apart; a k-step of 16
                    // dims is 32 bytes along the row
                    const uint64_t k_desc = umma_desc(base + slot * kItemBytes, 16, 1024, 2);
#pragma unroll
                    for (int u = 0; u < kUnits * kStreams; ++u) {
                        const int h = u / kStreams, s = u % kStreams, buf = buffer_of(g, s, h), use = use_of(g);
                        if (item == 0 && use >= 1)             // the weights that lie in the buffer have been used
                            fine = fine && __all_sync(0xffffffffu, tree_wait(misc + kTreeBarPvDone + buf * 8, (use - 1) & 1));
                        if (!fine) break;
                        tc_fence_after();
                        const uint64_t q_desc = umma_desc(q_smem + s * Geo::kQBytes, 16, 1024, 2);
                        if (elect_one()) {
#pragma unroll
                            for (int ks = 0; ks < 4 * kItemPanels; ++ks)
                                tc_mma_f16(tmem + buf * kUnit,
                                           q_desc + (uint64_t)(((item * kItemPanels + (ks >> 2)) * kTreePanelBytes + (ks & 3) * 32) >> 4),
                                           k_desc + (uint64_t)(((ks >> 2) * kTreePanelBytes + h * kUnit * 128 + (ks & 3) * 32) >> 4), idesc,
                                           item > 0 || ks > 0);
                            if (item + 1 == kItems) tc_commit(misc + kTreeBarSFull + buf * 8);
                            if (u + 1 == kUnits * kStreams) {
                                tc_commit(misc + kTreeBarKEmpty + slot * 8);
                                if (item + 1 == kItems && j + 1 == seg.t1) tc_commit(misc + kTreeBarQEmpty);
                            }
                        }
                        __syncwarp();
                    }
                }
            }
        }
        if (!fine && lane == 0 && a.status) atomicOr(a.status, kFlagCopyTimeout);
    } else if (warp == kWarpOutput) {
        // ================================ output MMAs ================================
        constexpr unsigned idesc = umma_idesc(128, kItemPanels * 64, 0, 1);       // weights K-major, V MN-major
        bool fine = true;
        int g = 0;
        for (int k = 0; fine; ++k) {
            fine = queue.wait(k);
            if (!fine) break;
            const TreeSegment seg = queue.entry(k);
            queue.done(k, lane);
            if (seg.b < 0) break;
            for (int j = seg.t0; j < seg.t1 && fine; ++j, ++g) {
#pragma unroll
                for (int u = 0; u < kUnits * kStreams; ++u) {
                    const int h = u / kStreams, s = u % kStreams, buf = buffer_of(g, s, h);
                    fine = fine && __all_sync(0xffffffffu, tree_wait(misc + kTreeBarPFull + buf * 8, use_of(g) & 1));
#pragma unroll
                    for (int item = 0; item < kItems; ++item) {
                        const int n = g * kItems + item, slot = n % kVSlots;
                        if (u == 0 && fine)
                            fine = __all_sync(0xffffffffu, tree_wait(misc + kTreeBarVFull + slot * 8, (n / kVSlots) & 1));
                        if (!fine) break;
                        tc_fence_after();
                        // 64-dim panels kTreePanelBytes apart, 8-token groups 1024 bytes apart; a k-step is
                        // 16 tokens = 2048 bytes.  Weights of 32 tokens: 16 columns of high, 16 of low parts.
                        const uint64_t v_desc = umma_desc(base + Ring::kVOffset + slot * kItemBytes, kTreePanelBytes, 1024, 2);
                        if (elect_one()) {
                            const unsigned acc = tmem + Geo::kOColumn + s * D + item * 128, weights = tmem + buf * kUnit;
#pragma unroll
                            for (int ks = 0; ks < kUnit / 16; ++ks) {
                                const unsigned at = weights + (ks >> 1) * 32 + (ks & 1) * 8;
                                const uint64_t v_step = v_desc + (uint64_t)(((h * (kUnit / 16) + ks) * 2048) >> 4);
                                tc_mma_f16_ts(acc, at, v_step, idesc, j > seg.t0 || h > 0 || ks > 0);
                                tc_mma_f16_ts(acc, at + 16, v_step, idesc, 1);
                            }
                            if (u + 1 == kUnits * kStreams) tc_commit(misc + kTreeBarVEmpty + slot * 8);
                            if (item + 1 == kItems) tc_commit(misc + kTreeBarPvDone + buf * 8);
                        }
                        __syncwarp();
                    }
                    if (!fine) break;
                }
            }
        }
        if (!fine && lane == 0 && a.status) atomicOr(a.status, kFlagCopyTimeout);
    } else {
        // ================================ softmax and epilogue ================================
        const int s = kStreams == 1 ? 0 : warp >> 2;                  // this warp's stream
        const int t = threadIdx.x & 127;                              // row of the block of rows = lane of tensor memory
        const unsigned lanes = (unsigned)((warp & 3) * 32) << 16;
        const unsigned acc = tmem + lanes + Geo::kOColumn + s * D;
        const int node_in_block = t / p.group, head = t - node_in_block * p.group;
        const bool used_row = node_in_block < p.nodes_per_block;
        const float factor = fabsf(a.scale_log2e), sign = copysignf(1.f, a.scale_log2e);
        bool fine = true;
        int g = 0;
        for (int k = 0;; ++k) {
            if (!fine || !queue.wait(k)) {
                fine = false;
                break;
            }
            const TreeSegment seg = queue.entry(k);
            queue.done(k, lane);
            if (seg.b < 0) break;
            const int node = (seg.rb * kStreams + s) * p.nodes_per_block + node_in_block;
            const bool exists = used_row && node < p.tree.tokens, live = exists && node < seg.nodes;
            const int prefix = seg.prefix();
            unsigned *poison = reinterpret_cast<unsigned *>(misc_ptr + kTreePoison) + (k & 7) * 4;
            // (the words of four segments ahead: no warp is more than two segments from another)
            if (threadIdx.x < 4) reinterpret_cast<volatile unsigned *>(misc_ptr + kTreePoison)[((k + 4) & 7) * 4 + threadIdx.x] = 0u;
            TreeRow row = {0, 0, live};
            if (live && seg.t1 * kTreeTile > prefix) row = tree_row(p.tree, seg.b, node, seg.nodes);
            // The reference is a logit before it is scaled, taken off before the scale comes in: the largest logit's
            // weight is exactly kGroupWeightScale then, however large it is.  l and the accumulator carry that scale.
            float m = kMinusHuge, l = 0.f;
            for (int j = seg.t0; j < seg.t1; ++j, ++g) {
                const int start = j * kTreeTile;
                const bool masked = start + kTreeTile > prefix;       // uniform
                // (stream 0 cleans for both: the output MMAs of a tile start with it)
                if (masked && s == 0) {
                    // Whether a value tile has landed is a parity of its slot's barrier: only once the slot's last tenant
                    // has landed does it speak of this tile.  This warp has seen logits of the tile before, for whose
                    // buffer the weights two tiles further back were used up; a tenant younger than that (head size 256:
                    // three slots for two items a tile) is waited for through the output MMAs that read it.
                    if constexpr (kVSlots < 3 * kItems) {
                        if (g > 0 && fine) fine = tree_wait(misc + kTreeBarPvDone + buffer_of(g - 1, s, kUnits - 1) * 8, use_of(g - 1) & 1);
                        fine = __all_sync(0xffffffffu, fine);
                    }
                    copies.template clean_values<32>(seg, j, g, (warp & 3) * 32, poison, fine);
                }
                // What the row sees of the tile, where that is not all of it; a negative scale takes the same way:
                // its sign goes to the logits, so that the maximum is the maximum.
                const bool special = masked || a.scale_log2e < 0.f;   // uniform
                Bits128 sees = {~(uint64_t)0, ~(uint64_t)0};
                if (masked) {
                    sees = {row.lo, row.hi};
                    if (start < prefix) {
                        const int n = prefix - start;                 // 1 .. 127 tokens before the tree
                        sees = sees.shifted_up(n);
                        if (row.all) {
                            sees.lo |= n >= 64 ? ~(uint64_t)0 : ((uint64_t)1 << n) - 1;
                            if (n > 64) sees.hi |= ((uint64_t)1 << (n - 64)) - 1;
                        }
                    } else {
                        sees = sees.shifted_down(start - prefix);
                    }
                }
                auto adjust = [&](float (&x)[32], int i) {
                    const unsigned word = sees.word(i);
#pragma unroll
                    for (int c = 0; c < 32; ++c) x[c] = word >> c & 1u ? x[c] * sign : -INFINITY;
                };
#pragma unroll 1
                for (int h = 0; h < kUnits; ++h) {
                    const int buf = buffer_of(g, s, h);
                    const unsigned logits = tmem + lanes + buf * kUnit;
                    if (fine) fine = tree_wait(misc + kTreeBarSFull + buf * 8, use_of(g) & 1);
                    fine = __all_sync(0xffffffffu, fine);
                    tc_fence_after();
                    float x[32], y[32];
                    float top = -INFINITY;
                    if constexpr (kUnit == 64) {
                        tc_issue_load32(x, logits);
                        tc_issue_load32(y, logits + 32);
                        tc_loaded32(x);
                        tc_loaded32(y);
                        if (special) {
                            adjust(x, 2 * h);
                            adjust(y, 2 * h + 1);
                        }
                        top = max32(y, max32(x, top));
                    } else {
                        // The row is read twice, 32 columns at a time in short loops, the next columns on their way while
                        // these are worked on: all 128 logits held at once leave no registers for anything else.
                        tc_issue_load32(x, logits);
#pragma unroll 1
                        for (int i = 0; i < 4; i += 2) {
                            tc_loaded32(x);
                            tc_issue_load32(y, logits + i * 32 + 32);
                            if (special) adjust(x, i);
                            top = max32(x, top);
                            tc_loaded32(y);
                            tc_issue_load32(x, logits + (i * 32 + 64) % 128);      // (the last one is the second pass's first)
                            if (special) adjust(y, i + 1);
                            top = max32(y, top);
                        }
                    }
                    // The reference follows the maximum lazily: weights stay below 2^kGroupLag.
                    const float rise = (top - m) * factor;
                    const bool moved = rise > kGroupLag;
                    if (__any_sync(0xffffffffu, moved)) {
                        const float alpha = moved ? fast_exp2(-rise) : 1.f;
                        if (moved) m = top;
                        l *= alpha;
                        if (j > seg.t0 || h > 0) {
                            // the accumulator holds the units before this one once their MMAs are complete
                            const int before = h > 0 ? g : g - 1;
                            if (fine) fine = tree_wait(misc + kTreeBarPvDone + buffer_of(before, s, h > 0 ? h - 1 : kUnits - 1) * 8, use_of(before) & 1);
                            fine = __all_sync(0xffffffffu, fine);
                            tc_fence_after();
#pragma unroll 1
                            for (int c0 = 0; c0 < D; c0 += 32) {
                                float o[32];
                                unsigned back[32];
                                tc_issue_load32(o, acc + c0);
                                tc_loaded32(o);
#pragma unroll
                                for (int c = 0; c < 32; ++c) back[c] = __float_as_uint(o[c] * alpha);
                                tc_store32(acc + c0, back);
                            }
                        }
                    }
                    // Weights (scaled by kGroupWeightScale inside the exponent), their sum, and their fp16 high and
                    // low parts over the logits: 16 + 16 columns per 32 tokens.
                    const float2 minus_ref = make_float2(-m, -m), factors = make_float2(factor, factor);
                    const float2 extra = make_float2(kGroupWeightLog2, kGroupWeightLog2);
                    float2 sum = make_float2(0.f, 0.f), sum_odd = make_float2(0.f, 0.f);
                    auto weigh = [&](const float (&z)[32], int i) {
                        unsigned parts[32];
#pragma unroll
                        for (int c = 0; c < 16; ++c) {
                            const float2 e = fma2(add2(make_float2(z[2 * c], z[2 * c + 1]), minus_ref), factors, extra);
                            const float2 w = make_float2(fast_exp2(e.x), fast_exp2(e.y));
                            float2 &total = c & 1 ? sum_odd : sum;
                            total = add2(total, w);
                            parts[c] = pack_half2(w.x, w.y);
                            const float2 back = __half22float2(*reinterpret_cast<const __half2 *>(&parts[c]));
                            const float2 rest = fma2(back, make_float2(-1.f, -1.f), w);
                            parts[16 + c] = pack_half2(rest.x, rest.y);
                        }
                        tc_store32(logits + i * 32, parts);
                    };
                    if constexpr (kUnit == 64) {
                        weigh(x, 0);
                        weigh(y, 1);
                    } else {
#pragma unroll 1
                        for (int i = 0; i < 4; i += 2) {
                            tc_loaded32(x);
                            tc_issue_load32(y, logits + i * 32 + 32);
                            if (special) adjust(x, i);
                            weigh(x, i);
                            tc_loaded32(y);
                            if (i == 0) tc_issue_load32(x, logits + 64);
                            if (special) adjust(y, i + 1);
                            weigh(y, i + 1);
                        }
                    }
                    l += (sum.x + sum.y) + (sum_odd.x + sum_odd.y);
                    tc_stored();
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbarrier_arrive(misc + kTreeBarPFull + buf * 8);
                }
            }
            // ---- the segment's end: the accumulator divided by the sum, to the output or the workspace ----
            if (fine) fine = tree_wait(misc + kTreeBarPvDone + buffer_of(g - 1, s, kUnits - 1) * 8, use_of(g - 1) & 1);
            fine = __all_sync(0xffffffffu, fine);
            tc_fence_after();
            const bool empty = !live || l == 0.f;                     // (a NaN sum is not an empty row's)
            const float inverse = empty ? 0.f : 1.f / l;
            const float lse2 = empty ? kMinusHuge : log2f(l) + fmaf(m, factor, -kGroupWeightLog2);
            const int64_t out_row = ((int64_t)seg.b * p.tree.tokens + node) * ((int64_t)a.heads * p.group) + (int64_t)seg.hk * p.group + head;
            const int64_t slot_row = (int64_t)seg.slot * p.item_rows + s * p.nodes_per_block * p.group + t;
            const bool whole = seg.whole();
            const volatile unsigned *taken = poison;
            const bool stray = live && (taken[0] | taken[1] | taken[2] | taken[3]) != 0u;
#pragma unroll 1
            for (int c0 = 0; c0 < D; c0 += 32) {
                float o[32];
                tc_issue_load32(o, acc + c0);
                tc_loaded32(o);
                if (exists && fine) {
#pragma unroll
                    for (int c = 0; c < 32; ++c) o[c] = empty ? 0.f : o[c] * inverse;
                    if (stray) {
                        float more[32];
                        for (int c = 0; c < 32; ++c) more[c] = 0.f;
                        tree_add_poisoned(a, seg, row, poison, out_row, D, c0, lse2, more);
#pragma unroll
                        for (int c = 0; c < 32; ++c) o[c] += more[c];
                    }
                    // (a thread's stores are a row apart: 32 bytes each where the buffer allows it)
                    if (whole) {
                        unsigned h[16];
#pragma unroll
                        for (int c = 0; c < 16; ++c) h[c] = pack_half2(o[2 * c], o[2 * c + 1]);
                        store_row<16>(a.out + out_row * D + c0, h);
                    } else {
                        unsigned w[32];
#pragma unroll
                        for (int c = 0; c < 32; ++c) w[c] = __float_as_uint(o[c]);
                        store_row<32>(a.part_o + slot_row * D + c0, w);
                    }
                }
                __syncwarp();
            }
            if (exists && fine) {
                if (!whole) a.part_lse[slot_row] = lse2;
                else if (a.lse) a.lse[out_row] = empty ? -INFINITY : lse2 * kLn2;
            }
            tc_fence_before();                                        // the accumulator has been read: the next tile may overwrite it
        }
        if (!fine && lane == 0 && a.status) atomicOr(a.status, kFlagCopyTimeout);
    }

    // ---- teardown: everyone is done with tensor memory before it is released ----
    tc_fence_before();
    __syncthreads();
    if (warp == kWarpLogits) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" :: "r"(tmem), "n"(512) : "memory");
    }
}

}  // namespace instinfer
