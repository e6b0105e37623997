// Decode attention over a latent cache for more than 32 query rows, by pairs of SMs, for sm_100a.
//
// The arithmetic and the split of the work are those of latent_kernels.cuh; here the ROWS are the long side of the MMAs:
// 128 of them, 64 in each block of a cluster of two, whose tensor cores work on one MMA together (cta_group::2):
//   S[128 rows x 128 tokens] = Q[128 x (L + 64)] tile^T       each block holds its rows' queries and half of the tile's tokens
//   O[128 rows x L]         += P[128 x 128] tile[128 x L]     each block holds its rows' weights and half of the tile's dims
// Why: one block cannot hold 128 rows (their queries are 144 KiB, their output all of tensor memory), and two blocks
// with 64 rows each, which the other form takes, read every operand out of shared memory at two thirds of the MMAs' rate and
// wait for a ring of two tiles.  Here the blocks share what they read, so that the MMAs run at their own rate; the price is that a
// block fetches the tile's other half of tokens once more for its half of the dims (1.9 x the bytes, of which the
// second ones come from L2).  Tensor memory holds two logit buffers of 64 columns and the output's L / 2: rows
// 0 .. 63 of a block are lanes 0 .. 63 with the first half of an MMA's columns and lanes 64 .. 127 with the second, so thread t of
// the softmax warps has row t % 64 and the tokens of half t / 64.
//
// Warps of a block: four of softmax; two that copy, keys ([64 tokens x 64 dims] panels) and values ([64 tokens x 128 dims]),
// into a ring each; and, in the first block, the two MMA issuers.  What the MMAs wait for is signalled to the first block's
// mbarriers (copies of both blocks complete there), what they complete is signalled to both blocks'.  Both blocks find the same
// segments by themselves.  Value rows that must not meet a weight of 0 (behind the sequence, or new tokens' rows that are not
// finite) are cleared by the copying warp, which lets the copies of such a tile land in its own block first.
//
// Measured: 128 rows, 32 sequences of 4k to 8k tokens 85 us (640 TFLOP/s), trees of 8 nodes x 16 heads over 7 sequences of up to 30k
// 70 us.  A tile takes 2.3 us of which its MMAs are 1.7 (a quarter of that for the weights' low parts): the logits wait for
// keys, since a whole tile of them has no room beside the rest.
//
// Every wait is bounded by the clock, as in the other kernels; one that runs out sets kFlagCopyTimeout.
#pragma once

#include "latent_kernels.cuh"

namespace instinfer {

constexpr int kPairTile = 128;                           // tokens per tile
constexpr int kPairRows = 64;                            // rows of a block
constexpr int kPairPanel = 64 * 128;                     // 64 tokens or rows of 64 dims (or 64 tokens' weights of 64 rows)
constexpr int kPairThreads = 256;
constexpr int kPairWarpKeys = 4, kPairWarpValues = 5, kPairWarpLogits = 6, kPairWarpOutput = 7;

// Offsets inside the misc region.
constexpr int kPairBarKFull = 0;       // [8] of the first block: both blocks' part of an item landed
constexpr int kPairBarKEmpty = 64;     // [8]
constexpr int kPairBarVFull = 128;     // [2] of the first block: the values of a half of the tokens
constexpr int kPairBarVOwn = 144;      // [2] this block's part of them landed (where its rows are looked at)
constexpr int kPairBarSFull = 320;     // [2]
constexpr int kPairBarSFree = 336;     // [2] of the first block
constexpr int kPairBarPFull = 224;     // [2] of the first block: the weights of a half of the tokens
constexpr int kPairBarPvDone = 240;    // [2] the MMAs that read those weights and values are complete
constexpr int kPairBarQFull = 368;     // of the first block
constexpr int kPairBarQEmpty = 376;
constexpr int kPairBarSegFull = 384;   // [4]
constexpr int kPairBarSegEmpty = 416;  // [4]
constexpr int kPairTmemPtr = 448;
constexpr int kPairTotal = 452;        // see latent_scan
constexpr int kPairScan = 464;
constexpr int kPairSegments = 528;     // [4] LatentSegment
constexpr int kPairExchange = 752;     // [128] floats: a thread's number for the thread with the same row's other half
constexpr int kPairMiscBytes = 752 + 512;
static_assert(kPairScan - kPairTotal == kLatScan - kLatTotal && kPairSegments + 4 * kLatSegmentBytes <= kPairExchange, "misc region");

template <int L>
struct PairGeometry {
    static_assert(L == 512, "instances");
    static constexpr int kPanels = L / 64 + 1;                           // key panels of a tile, the turned part the last
    static constexpr int kParts = L / 256;                               // 128-dim parts of a block's half of the dims
    // Large items, because an item's wait and commit cost the issuers 0.2 us whatever its size (with keys by the panel that
    // took longer than the MMAs): keys by three panels, values by halves of the tile's tokens.
    static constexpr int kKeyPanels = 3, kKeyItems = (kPanels + kKeyPanels - 1) / kKeyPanels, kKSlots = 2;
    static constexpr int kValuePanels = 2 * kParts, kItemBytes = kValuePanels * kPairPanel;
    static constexpr int kVOffset = kKSlots * kKeyPanels * kPairPanel;
    static constexpr int kQOffset = kVOffset + 2 * kItemBytes;
    static constexpr int kQBytes = kPanels * kPairPanel;
    static constexpr int kPOffset = kQOffset + kQBytes;                  // high parts [half of the tokens], then low parts
    static constexpr int kMiscOffset = kPOffset + 4 * kPairPanel;
    static constexpr int kSmemBytes = kMiscOffset + kPairMiscBytes + 1024;
    static constexpr int kOColumn = 128;                                 // two logit buffers of 64 columns, then the output
    static constexpr int kTmemCols = 512;
    static_assert(kOColumn + (kParts - 1) * 128 + 256 <= kTmemCols, "tensor memory");
    static_assert(kSmemBytes <= 227 * 1024, "one block per SM must fit");
};

// ---- what a pair needs besides the wrappers of one block ----
__device__ __forceinline__ unsigned of_first_block(unsigned addr)          // the same place in the cluster's first block
{
    unsigned there;
    asm volatile("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(there) : "r"(addr));
    return there;
}
__device__ __forceinline__ void pair_arrive(unsigned bar)                  // bar: of_first_block
{
    asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" :: "r"(bar) : "memory");
}
__device__ __forceinline__ void pair_expect_bytes(unsigned bar, unsigned bytes)
{
    asm volatile("mbarrier.arrive.expect_tx.shared::cluster.b64 _, [%0], %1;" :: "r"(bar), "r"(bytes) : "memory");
}
__device__ __forceinline__ void pair_mma_f16(unsigned d_tmem, uint64_t a_desc, uint64_t b_desc, unsigned idesc, unsigned accumulate)
{
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
                 "tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}"
                 :: "r"(d_tmem), "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(accumulate) : "memory");
}
__device__ __forceinline__ void pair_commit(unsigned bar)                  // arrives on `bar` of both blocks
{
    asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;"
                 :: "r"(bar), "h"((unsigned short)3) : "memory");
}
// Into this block's memory; the bytes are reported to the first block's barrier (bar: of_first_block).
__device__ __forceinline__ void pair_load_2d(unsigned dst, const CUtensorMap *map, int x, int y, unsigned bar)
{
    asm volatile("cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes "
                 "[%0], [%1, {%2, %3}], [%4];"
                 :: "r"(dst), "l"(reinterpret_cast<uint64_t>(map)), "r"(x), "r"(y), "r"(bar) : "memory");
}
__device__ __forceinline__ void pair_load_3d(unsigned dst, const CUtensorMap *map, int x, int y, int z, unsigned bar)
{
    asm volatile("cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes "
                 "[%0], [%1, {%2, %3, %4}], [%5];"
                 :: "r"(dst), "l"(reinterpret_cast<uint64_t>(map)), "r"(x), "r"(y), "r"(z), "r"(bar) : "memory");
}

template <typename E, int L>
__global__ void __launch_bounds__(kPairThreads, 1)
latent_pair_kernel(const __grid_constant__ LatentParams p, const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_cache)
{
    using Geo = PairGeometry<L>;
    constexpr int kPanels = Geo::kPanels, kParts = Geo::kParts, kKeyPanels = Geo::kKeyPanels, kKeyItems = Geo::kKeyItems, kKSlots = Geo::kKSlots;
    constexpr unsigned kTypes = std::is_same<E, __half>::value ? 0u : 1u << 7 | 1u << 10;
    extern __shared__ unsigned char smem_raw[];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, rank = blockIdx.x & 1;       // (clusters of two consecutive blocks)
    allow_next_kernel();
    wait_for_previous_kernels();

    const unsigned raw = static_cast<unsigned>(__cvta_generic_to_shared(smem_raw));
    const unsigned base = (raw + 1023u) & ~1023u;
    unsigned char *smem = smem_raw + (base - raw);
    const unsigned q_smem = base + Geo::kQOffset, p_smem = base + Geo::kPOffset, misc = base + Geo::kMiscOffset, first_misc = of_first_block(misc);
    unsigned char *misc_ptr = smem + Geo::kMiscOffset;
    auto entry = [&](int k) -> LatentSegment & { return reinterpret_cast<LatentSegment *>(misc_ptr + kPairSegments)[k & 3]; };
    auto wait_segment = [&](int k) -> bool { return __all_sync(0xffffffffu, tree_wait(misc + kPairBarSegFull + (k & 3) * 8, (k >> 2) & 1)); };
    auto done_segment = [&](int k) {
        __syncwarp();
        if (lane == 0) mbarrier_arrive(misc + kPairBarSegEmpty + (k & 3) * 8);
    };

    LatentFinder finder;               // (of the key-copying warp)
    const int pair = blockIdx.x >> 1;
    finder.plane = pair % p.planes;
    finder.team = pair / p.planes;
    finder.items = latent_plane_items(p, finder.plane);
    finder.w0 = finder.start = 0;
    if (p.batch > 32) latent_scan(p, misc_ptr + (kPairTotal - kLatTotal), kPairThreads, finder.plane, finder.items, finder.team);
    LatentSegment seg;
    if (warp == kPairWarpLogits) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;"
                     :: "r"(misc + kPairTmemPtr), "n"(Geo::kTmemCols) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    } else if (warp == kPairWarpKeys && p.batch <= 32) {
        if (lane < 2) asm volatile("prefetch.tensormap [%0];" :: "l"(reinterpret_cast<uint64_t>(lane ? &map_cache : &map_q)) : "memory");
        finder.load(p, lane);
        if (blockIdx.x == 0 && lane < p.batch) {                  // lengths out of range
            int nodes;
            (void)checked_tree(p.tree, p.seq_lens, p.max_seq_len, p.status, lane, true, nodes);
        }
        finder.begin(p, __shfl_sync(0xffffffffu, finder.stop, 31));
        seg = finder.template next<E, L>(p, lane);
    } else if (warp == kPairWarpOutput && lane == 0) {
        for (int s = 0; s < 8; ++s) {
            mbarrier_init(misc + kPairBarKFull + s * 8, 2);       // both blocks' copying warps
            mbarrier_init(misc + kPairBarKEmpty + s * 8, 1);
        }
        for (int s = 0; s < 2; ++s) {
            mbarrier_init(misc + kPairBarVFull + s * 8, 2);
            mbarrier_init(misc + kPairBarVOwn + s * 8, 1);
            mbarrier_init(misc + kPairBarSFull + s * 8, 1);
            mbarrier_init(misc + kPairBarSFree + s * 8, 8);       // both blocks' softmax warps
            mbarrier_init(misc + kPairBarPFull + s * 8, 4);       // those of one half of the tokens
            mbarrier_init(misc + kPairBarPvDone + s * 8, 1);
        }
        mbarrier_init(misc + kPairBarQFull, 2);
        mbarrier_init(misc + kPairBarQEmpty, 1);
        for (int s = 0; s < 4; ++s) {
            mbarrier_init(misc + kPairBarSegFull + s * 8, 1);
            mbarrier_init(misc + kPairBarSegEmpty + s * 8, rank == 0 ? 7 : 5);    // softmax, the other copying warp, the MMA issuers
        }
        mbarrier_init_fence();
    }
    tc_fence_before();
    __syncthreads();
    // the other block's barriers are ready and its tensor memory is its own
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
    tc_fence_after();
    const unsigned tmem = *reinterpret_cast<volatile unsigned *>(misc_ptr + kPairTmemPtr);

    const bool paged = p.block_table != nullptr;
    const int T = p.run_tokens;
    // lane i: the cache row at which run i of tokens [start, start + 64) of a sequence starts, -1: not a run of it, -2: not readable
    auto run_row = [&](int b, int len, int start) -> int {
        if (start + lane * T >= len || lane * T >= 64) return -1;
        if (!paged) return b * p.s_max + start;           // (T = 64; rows past the tensor's end read as zeros)
        const int idx = (start + lane * T) / p.block_tokens;
        if (!bounds_ok(idx < p.max_blocks_per_seq, p.status)) return -2;
        const int phys = p.block_table[(int64_t)b * p.max_blocks_per_seq + idx];
        if (phys < 0 || (int64_t)phys >= p.num_phys_blocks) {
            if (p.status) atomicOr(p.status, kFlagBlockRange);
            return -2;
        }
        const int row = phys * p.block_tokens + (start + lane * T) % p.block_tokens;      // (< 2^31: checked by the host)
        return bounds_ok((int64_t)row + T <= p.cache_rows, p.status) ? row : -2;
    };
    // What a warp copies of 64 tokens, whose runs' rows run_row has: lane r + 8 q asks for panel q of run r.
    struct Rows {
        int row;                      // this lane's run's, or negative
        unsigned bytes;               // of one panel
        bool missing, any_missing;    // (of the runs, lane by lane) blocks that cannot be read count as zeros
    };
    auto rows_of = [&](int runs) -> Rows {
        Rows rows;
        rows.bytes = __popc(__ballot_sync(0xffffffffu, runs >= 0)) * (unsigned)(T * 128);
        rows.missing = runs == -2;
        rows.any_missing = __any_sync(0xffffffffu, rows.missing);
        rows.row = __shfl_sync(0xffffffffu, runs, lane & 7);
        return rows;
    };
    // `panels` (up to 4) panels of 64 dims from `dim` on; the bytes go to bar, of the first block or (own) this one.
    auto copy_rows = [&](const Rows &rows, unsigned dst_offset, int dim, int panels, unsigned bar, bool own) {
        if (rows.any_missing) {
            if (rows.missing) {
                const uint4 zero = make_uint4(0u, 0u, 0u, 0u);
#pragma unroll 1
                for (int i = 0; i < panels * T * 8; ++i)
                    *reinterpret_cast<uint4 *>(smem + dst_offset + i / (T * 8) * kPairPanel + lane * T * 128 + i % (T * 8) * 16) = zero;
                fence_async_proxy();
            }
            __syncwarp();
        }
        if (lane == 0) {
            if (own) mbarrier_expect_bytes(bar, rows.bytes * panels);
            else pair_expect_bytes(bar, rows.bytes * panels);
        }
        __syncwarp();
        if (rows.row >= 0 && lane < 8 * panels) {
            const unsigned to = base + dst_offset + (lane >> 3) * kPairPanel + (lane & 7) * T * 128;
            if (own) tma_load_2d(to, &map_cache, dim + (lane >> 3) * 64, rows.row, bar);
            else pair_load_2d(to, &map_cache, dim + (lane >> 3) * 64, rows.row, bar);
        }
    };

    // A copying warp whose wait ran out: copies in flight get some milliseconds to land before shared memory is handed on.
    auto give_up = [&]() {
        if (lane == 0 && p.status) atomicOr(p.status, kFlagCopyTimeout);
        for (const long long start = clock64(); clock64() - start < 8000000ll;) __nanosleep(1000);
    };

    if (warp == kPairWarpKeys) {
        // ================================ copies of keys and queries ================================
        if (p.batch > 32) {
            const int *found = reinterpret_cast<const int *>(misc_ptr + kPairTotal);
            finder.begin(p, found[0]);
            if (finder.tile < finder.end) {
                finder.w0 = found[1];
                finder.start = found[2];
                finder.load(p, lane);
            }
            seg = finder.template next<E, L>(p, lane);
        }
        int n = 0, k = 0;                                 // items and segments so far
        bool fine = true;
        auto announce = [&](const LatentSegment &s, int i) -> bool {
            if (i >= 4 && !__all_sync(0xffffffffu, tree_wait(misc + kPairBarSegEmpty + (i & 3) * 8, ((i >> 2) - 1) & 1))) return false;
            if (lane == 0) {
                entry(i) = s;
                mbarrier_arrive(misc + kPairBarSegFull + (i & 3) * 8);
            }
            return true;
        };
        (void)announce(seg, 0);
        // Rows of this tile, the next and the one after it: block ids are asked for two tiles ahead, and the next tile is
        // brought into L2 while this one is copied, so that a panel's slot waits for L2's latency and not for memory's.
        int rows = -1, rows_next = -1;
        if (seg.b >= 0) {
            rows = run_row(seg.b, seg.len, seg.t0 * kPairTile + rank * 64);
            if (seg.t0 + 1 < seg.t1) rows_next = run_row(seg.b, seg.len, (seg.t0 + 1) * kPairTile + rank * 64);
        }
        for (; fine && seg.b >= 0; ++k) {
            LatentSegment after = seg;
            int rows_after = -1, rows_after_next = -1;
            for (int j = seg.t0; j < seg.t1 && fine; ++j) {
                if (j == seg.t0) {
                    // the query rows wait for the last segment's logits
                    if (k >= 1) fine = __all_sync(0xffffffffu, tree_wait(misc + kPairBarQEmpty, (k - 1) & 1));
                    if (!fine) break;
                    const int half = (p.block_rows + 1) / 2;      // rows of the first block
                    if (lane == 0) pair_expect_bytes(first_misc + kPairBarQFull, (unsigned)Geo::kQBytes);
                    __syncwarp();
                    if (lane < kPanels)                           // (rows behind the sequence's last are zeros)
                        pair_load_3d(q_smem + lane * kPairPanel, &map_q, lane * 64, seg.row0 + rank * half, seg.b, first_misc + kPairBarQFull);
                    __syncwarp();
                }
                const int now = rows;
                rows = rows_next;
                rows_next = j + 2 < seg.t1 ? run_row(seg.b, seg.len, (j + 2) * kPairTile + rank * 64) : -1;
                latent_prefetch(p, rows, T, (L + kLatentRope) * 2);
                const Rows of_tile = rows_of(now);
#pragma unroll 1
                for (int item = 0; item < kKeyItems && fine; ++item) {
                    // (one answer for the warp: a copy has full-warp barriers, and its bytes are announced by one lane for all)
                    const int slot = n % kKSlots;
                    if (n >= kKSlots) fine = __all_sync(0xffffffffu, tree_wait(misc + kPairBarKEmpty + slot * 8, (n / kKSlots - 1) & 1));
                    if (fine)
                        copy_rows(of_tile, slot * kKeyPanels * kPairPanel, item * kKeyPanels * 64, min(kKeyPanels, kPanels - item * kKeyPanels),
                                  first_misc + kPairBarKFull + slot * 8, false);
                    ++n;
                }
                if (j > seg.t0 || !fine) continue;
                after = finder.template next<E, L>(p, lane);
                fine = announce(after, k + 1);
                if (after.b >= 0) {
                    rows_after = run_row(after.b, after.len, after.t0 * kPairTile + rank * 64);
                    if (after.t0 + 1 < after.t1) rows_after_next = run_row(after.b, after.len, (after.t0 + 1) * kPairTile + rank * 64);
                }
            }
            if (!fine) break;
            seg = after;
            rows = rows_after;
            rows_next = rows_after_next;
        }
        if (!fine) give_up();
    } else if (warp == kPairWarpValues) {
        // ================================ copies of values ================================
        int g = 0;
        unsigned own = 0;                                 // bit h: parity of the phase that half h's own barrier is in
        bool fine = true;
        for (int k = 0; fine; ++k) {
            fine = wait_segment(k);
            if (!fine) break;
            const int b = entry(k).b, len = entry(k).len, prefix = entry(k).prefix(), t0 = entry(k).t0, t1 = entry(k).t1;
            done_segment(k);
            if (b < 0) break;
            int rows0 = run_row(b, len, t0 * kPairTile), rows1 = run_row(b, len, t0 * kPairTile + 64);
            for (int j = t0; j < t1 && fine; ++j, ++g) {
                const int start = j * kPairTile;
                const Rows half0 = rows_of(rows0), half1 = rows_of(rows1);
                if (j + 1 < t1) {
                    rows0 = run_row(b, len, start + kPairTile);
                    rows1 = run_row(b, len, start + kPairTile + 64);
                }
                const bool looked_at = start + kPairTile > prefix;
#pragma unroll 1
                for (int half = 0; half < 2 && fine; ++half) {
                    if (g > 0) fine = __all_sync(0xffffffffu, tree_wait(misc + kPairBarPvDone + half * 8, (g - 1) & 1));
                    if (fine)
                        copy_rows(half == 0 ? half0 : half1, Geo::kVOffset + half * Geo::kItemBytes, rank * (L / 2), Geo::kValuePanels,
                                  looked_at ? misc + kPairBarVOwn + half * 8 : first_misc + kPairBarVFull + half * 8, looked_at);
                }
                if (!looked_at) continue;
                // The halves land here, and rows that must not meet a weight of 0 are cleared.
#pragma unroll 1
                for (int half = 0; half < 2 && fine; ++half) {
                    fine = __all_sync(0xffffffffu, tree_wait(misc + kPairBarVOwn + half * 8, own >> half & 1u));
                    if (!fine) break;
                    own ^= 1u << half;
                    static_assert(8 * Geo::kValuePanels == 32, "a lane has one chunk of a row");
                    const int first = start + half * 64;                   // row r of the half is position first + r
                    unsigned char *chunk = smem + Geo::kVOffset + half * Geo::kItemBytes + (lane >> 3) * kPairPanel + (lane & 7) * 16;
#pragma unroll 1
                    for (int r = max(0, prefix - first); r < 64; ++r) {
                        uint4 *at = reinterpret_cast<uint4 *>(chunk + r * 128);
                        if (first + r >= len || __any_sync(0xffffffffu, !latent_finite8<E>(*at))) *at = make_uint4(0u, 0u, 0u, 0u);
                    }
                    fence_async_proxy();
                    __syncwarp();
                    if (lane == 0) pair_arrive(first_misc + kPairBarVFull + half * 8);
                }
            }
        }
        if (!fine) give_up();
    } else if (warp == kPairWarpLogits) {
        // ================================ logit MMAs (of the first block) ================================
        constexpr unsigned idesc = umma_idesc(128, 128, 0, 0) | kTypes;    // queries and tile K-major
        const uint64_t q_desc = umma_desc(q_smem, 16, 1024, 2), k_desc = umma_desc(base, 16, 1024, 2);
        bool fine = rank == 0;
        int g = 0;
        for (int k = 0; fine; ++k) {
            fine = wait_segment(k);
            if (!fine) break;
            const int b = entry(k).b, t0 = entry(k).t0, t1 = entry(k).t1;
            done_segment(k);
            if (b < 0) break;
            fine = __all_sync(0xffffffffu, tree_wait(misc + kPairBarQFull, k & 1));
            for (int j = t0; j < t1 && fine; ++j, ++g) {
                const int buf = g & 1;
                if (g >= 2) fine = __all_sync(0xffffffffu, tree_wait(misc + kPairBarSFree + buf * 8, ((g >> 1) - 1) & 1));
#pragma unroll
                for (int item = 0; item < kKeyItems; ++item) {
                    const int n = g * kKeyItems + item, slot = n % kKSlots;
                    if (fine) fine = tree_wait(misc + kPairBarKFull + slot * 8, (n / kKSlots) & 1);
                    tc_fence_after();
                    const uint64_t item_desc = k_desc + (uint64_t)((slot * kKeyPanels * kPairPanel) >> 4);
                    // rows of 128 bytes, 8-row groups 1024 bytes apart; a k-step of 16 dims is 32 bytes along the row
                    if (elect_one() && fine) {
#pragma unroll
                        for (int ks = 0; ks < 4 * kKeyPanels; ++ks) {
                            const int panel = item * kKeyPanels + (ks >> 2), at = (ks & 3) * 32;
                            if (panel < kPanels)
                                pair_mma_f16(tmem + buf * 64, q_desc + (uint64_t)((panel * kPairPanel + at) >> 4),
                                             item_desc + (uint64_t)(((ks >> 2) * kPairPanel + at) >> 4), idesc, item > 0 || ks > 0);
                        }
                        pair_commit(misc + kPairBarKEmpty + slot * 8);
                        if (item + 1 == kKeyItems) {
                            pair_commit(misc + kPairBarSFull + buf * 8);
                            if (j + 1 == t1) pair_commit(misc + kPairBarQEmpty);
                        }
                    }
                    __syncwarp();
                }
                fine = __all_sync(0xffffffffu, fine);
            }
        }
        if (!fine && rank == 0 && lane == 0 && p.status) atomicOr(p.status, kFlagCopyTimeout);
    } else if (warp == kPairWarpOutput) {
        // ================================ output MMAs (of the first block) ================================
        constexpr unsigned idesc = umma_idesc(128, 256, 0, 1) | kTypes;    // weights K-major, tile MN-major
        // weights: as the queries; tile: its 64-dim panels kPairPanel apart, 8-token groups 1024 bytes apart, a k-step of 16 tokens
        // is 32 bytes of a weights' row and 2048 bytes of the tile
        const uint64_t p_desc = umma_desc(p_smem, 16, 1024, 2), v_desc = umma_desc(base + Geo::kVOffset, kPairPanel, 1024, 2);
        bool fine = rank == 0;
        int g = 0;
        for (int k = 0; fine; ++k) {
            fine = wait_segment(k);
            if (!fine) break;
            const int b = entry(k).b, t0 = entry(k).t0, t1 = entry(k).t1;
            done_segment(k);
            if (b < 0) break;
            for (int j = t0; j < t1 && fine; ++j, ++g) {
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    if (fine) fine = tree_wait(misc + kPairBarVFull + half * 8, g & 1);
                    if (fine) fine = tree_wait(misc + kPairBarPFull + half * 8, g & 1);
                    tc_fence_after();
                    if (elect_one() && fine) {
#pragma unroll
                        for (int part = 0; part < kParts; ++part) {
#pragma unroll
                            for (int ks = 0; ks < 8; ++ks)                 // the high parts, then the low parts
                                pair_mma_f16(tmem + Geo::kOColumn + part * 128, p_desc + (uint64_t)(((ks >> 2) * 2 * kPairPanel + half * kPairPanel + (ks & 3) * 32) >> 4),
                                             v_desc + (uint64_t)((half * Geo::kItemBytes + part * 2 * kPairPanel + (ks & 3) * 2048) >> 4), idesc,
                                             j > t0 || half > 0 || ks > 0);
                        }
                        pair_commit(misc + kPairBarPvDone + half * 8);
                    }
                    __syncwarp();
                }
                fine = __all_sync(0xffffffffu, fine);
            }
        }
        if (!fine && rank == 0 && lane == 0 && p.status) atomicOr(p.status, kFlagCopyTimeout);
    } else {
        // ================================ softmax and epilogue ================================
        const int t = threadIdx.x, r = t & 63, side = t >> 6;              // this thread's row of the block, its half of the tokens (and dims)
        const unsigned lanes = tmem + ((unsigned)(warp * 32) << 16);
        float *exchange = reinterpret_cast<float *>(misc_ptr + kPairExchange);
        const int half_rows = (p.block_rows + 1) / 2, row = rank * half_rows + r;         // of the row block
        const bool my_row = r < half_rows && row < p.block_rows;
        const float scale = p.scale_log2e, sign = copysignf(1.f, scale), heads_inverse = 1.f / (float)p.q_heads;
        bool fine = true;
        int g = 0;
        for (int k = 0;; ++k) {
            if (group_any(1, !wait_segment(k) || !fine)) {
                fine = false;
                break;
            }
            const LatentSegment &seg = entry(k);
            if (seg.b < 0) break;
            const int nodes = seg.nodes, prefix = seg.prefix(), t0 = seg.t0, t1 = seg.t1;
            const int node = latent_node(seg.row0 + row, heads_inverse);
            const bool live = my_row && row < seg.rows && node < nodes;
            // the new tokens that this row sees: asked for here, looked at in the last tiles
            Bits128 sees = {0, 0};
            if (live && t1 * kPairTile > prefix) {
                if (p.tree.mask == nullptr) {
                    sees.lo = node >= 63 ? ~0ull : (1ull << (node + 1)) - 1;
                    sees.hi = node >= 127 ? ~0ull : node >= 64 ? (1ull << (node - 63)) - 1 : 0;
                } else {
                    const TreeRow bits = tree_row(p.tree, seg.b, node, nodes);
                    sees = {bits.lo, bits.hi};
                }
            }
            float offset = -kMinusHuge * sign;                             // the negated reference, a logit before the scale
            float2 l = make_float2(0.f, 0.f);
            for (int j = t0; j < t1; ++j, ++g) {
                const int buf = g & 1, start = j * kPairTile + side * 64;  // position of column 0
                const bool masked = (j + 1) * kPairTile > prefix;          // uniform
                uint64_t shown = ~0ull;                                    // this thread's tokens that its row sees
                if (masked) {
                    const int at = start - prefix;                         // column 0 as a new token
                    if (!live) shown = 0;
                    else if (at >= 0) shown = at < 128 ? sees.shifted_down(at).lo : 0;
                    else if (at > -64) shown = sees.lo << -at | ((1ull << -at) - 1);
                }
                if (fine) fine = tree_wait(misc + kPairBarSFull + buf * 8, (g >> 1) & 1);
                fine = __all_sync(0xffffffffu, fine);
                tc_fence_after();
                float x[32], y[32];
                tc_issue_load32(x, lanes + buf * 64);
                tc_issue_load32(y, lanes + buf * 64 + 32);
                for (int attempt = 0;; ++attempt) {
                    tc_loaded32(x);
                    tc_loaded32(y);
#pragma unroll
                    for (int i = 0; i < 32; i += 2) {
                        const float2 a = mul2(add2(make_float2(x[i], x[i + 1]), make_float2(offset, offset)), make_float2(scale, scale));
                        const float2 b = mul2(add2(make_float2(y[i], y[i + 1]), make_float2(offset, offset)), make_float2(scale, scale));
                        x[i] = a.x;
                        x[i + 1] = a.y;
                        y[i] = b.x;
                        y[i + 1] = b.y;
                    }
                    if (masked) {
#pragma unroll
                        for (int i = 0; i < 32; ++i) {
                            if (!((unsigned)shown >> i & 1u)) x[i] = -INFINITY;
                            if (!((unsigned)(shown >> 32) >> i & 1u)) y[i] = -INFINITY;
                        }
                    }
                    const float most = fmaxf(max32(x, -INFINITY), max32(y, -INFINITY));
                    if (attempt > 0 || !group_any(1, most > kGroupLag)) break;
                    // ---- some row's reference moves (rare after a segment's first tile) ----
                    if (j > t0) {                                          // the output holds the tiles before this one
                        if (fine) fine = tree_wait(misc + kPairBarPvDone + 8, (g - 1) & 1);
                        fine = __all_sync(0xffffffffu, fine);
                        tc_fence_after();
                    }
                    // (the largest logit again, from tensor memory: what is scaled has lost bits)
                    tc_issue_load32(x, lanes + buf * 64);
                    tc_issue_load32(y, lanes + buf * 64 + 32);
                    tc_loaded32(x);
                    tc_loaded32(y);
                    float top = -INFINITY;
#pragma unroll
                    for (int i = 0; i < 32; ++i) {
                        if (!masked || ((unsigned)shown >> i & 1u)) top = fmaxf(top, x[i] * sign);
                        if (!masked || ((unsigned)(shown >> 32) >> i & 1u)) top = fmaxf(top, y[i] * sign);
                    }
                    exchange[t] = top;
                    group_sync(2);
                    top = fmaxf(top, exchange[t ^ 64]);
                    group_sync(2);
                    float alpha = 1.f;                                     // 2^(old - new reference)
                    const float moved = -top * sign, rise = (offset - moved) * scale;
                    if (rise > kGroupLag) {
                        alpha = fast_exp2(-rise);
                        offset = moved;
                    }
                    l.x *= alpha;
                    l.y *= alpha;
                    if (j > t0 && __any_sync(0xffffffffu, alpha != 1.f)) {
#pragma unroll 1
                        for (int c0 = 0; c0 < L / 2; c0 += 16) {
                            float o[16];
                            tc_issue_load16(o, lanes + Geo::kOColumn + c0);
                            tc_loaded16(o);
#pragma unroll
                            for (int c = 0; c < 16; ++c) o[c] *= alpha;
                            tc_store16(lanes + Geo::kOColumn + c0, o);
                        }
                    }
                    tc_issue_load32(x, lanes + buf * 64);
                    tc_issue_load32(y, lanes + buf * 64 + 32);
                }
                tc_fence_before();
                __syncwarp();
                if (lane == 0) pair_arrive(first_misc + kPairBarSFree + buf * 8);
                unsigned hi[32], lo[32];                                   // pairs of weights
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const float2 a = make_float2(fast_exp2(x[2 * i]), fast_exp2(x[2 * i + 1])), b = make_float2(fast_exp2(y[2 * i]), fast_exp2(y[2 * i + 1]));
                    l = add2(l, add2(a, b));
                    split_weights<E>(a, hi[i], lo[i]);
                    split_weights<E>(b, hi[16 + i], lo[16 + i]);
                }
                if (g > 0 && fine) fine = tree_wait(misc + kPairBarPvDone + side * 8, (g - 1) & 1);      // the last tile's MMAs have read the weights
                unsigned char *to = smem + Geo::kPOffset + side * kPairPanel + r * 128;
#pragma unroll
                for (int c = 0; c < 8; ++c) {
                    const int at = (c ^ (r & 7)) * 16;                     // (128-byte swizzle)
                    *reinterpret_cast<uint4 *>(to + at) = make_uint4(hi[4 * c], hi[4 * c + 1], hi[4 * c + 2], hi[4 * c + 3]);
                    *reinterpret_cast<uint4 *>(to + 2 * kPairPanel + at) = make_uint4(lo[4 * c], lo[4 * c + 1], lo[4 * c + 2], lo[4 * c + 3]);
                }
                fence_async_proxy();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) pair_arrive(first_misc + kPairBarPFull + side * 8);
            }
            // ---- the segment's end: the row's sum, then the output divided by it ----
            float total = l.x + l.y;
            exchange[t] = total;
            group_sync(2);
            total = side == 0 ? total + exchange[t ^ 64] : exchange[t ^ 64] + total;
            const bool whole = seg.whole(), writes = my_row && row < seg.rows, empty = !live || total == 0.f;      // (a NaN sum is not an empty row's)
            if (writes && side == 0 && fine && seg.lse) seg.lse[row] = empty ? (whole ? -INFINITY : kMinusHuge) : fmaf(-offset, p.scale, logf(total));
            const float inverse = empty ? 0.f : __fdividef(1.f / kLatentWeightScale<E>, total);
            if (fine) fine = tree_wait(misc + kPairBarPvDone + 8, (g - 1) & 1);                // (the second half's are the last)
            fine = __all_sync(0xffffffffu, fine);
            tc_fence_after();
            // 32 dims of a warp's 32 rows at a time, through the weights' memory (nobody reads them now), so that what a warp
            // stores together are whole 128-byte pieces of four rows; the next dims are asked for meanwhile.
            unsigned char *stage = smem + Geo::kPOffset + warp * 4096;
            const int row_in_block = (warp & 1) * 32 + (lane >> 3);        // lane's first row; the others are 4, 8 .. further
            const int rows_left = fine ? min(half_rows, seg.rows - rank * half_rows) - row_in_block : 0;
            const int64_t to = (int64_t)(rank * half_rows + row_in_block) * L + side * (L / 2) + (lane & 7) * 4;
            E *rounded_out = static_cast<E *>(seg.out) + to;
            float *out = static_cast<float *>(seg.out) + to;
            const unsigned char *from = stage + (lane >> 3) * 128;
            float o[32];
            tc_issue_load32(o, lanes + Geo::kOColumn);
#pragma unroll 1
            for (int c0 = 0; c0 < L / 2; c0 += 32) {                       // dims side * L / 2 + c0 ..
                tc_loaded32(o);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    float4 four = make_float4(o[4 * i] * inverse, o[4 * i + 1] * inverse, o[4 * i + 2] * inverse, o[4 * i + 3] * inverse);
                    if (empty) four = make_float4(0.f, 0.f, 0.f, 0.f);     // (an empty row's output may hold anything)
                    *reinterpret_cast<float4 *>(stage + lane * 128 + (i ^ (lane & 7)) * 16) = four;
                }
                if (c0 + 32 < L / 2) tc_issue_load32(o, lanes + Geo::kOColumn + c0 + 32);
                __syncwarp();
                float4 fours[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) fours[i] = *reinterpret_cast<const float4 *>(from + i * 512 + ((lane & 7) ^ ((4 * i + (lane >> 3)) & 7)) * 16);
                if (whole) {
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const E rounded[4] = {latent_round<E>(fours[i].x), latent_round<E>(fours[i].y), latent_round<E>(fours[i].z), latent_round<E>(fours[i].w)};
                        if (4 * i < rows_left) *reinterpret_cast<uint2 *>(rounded_out + 4 * i * L + c0) = *reinterpret_cast<const uint2 *>(rounded);
                    }
                } else {
#pragma unroll
                    for (int i = 0; i < 8; ++i)
                        if (4 * i < rows_left) *reinterpret_cast<float4 *>(out + 4 * i * L + c0) = fours[i];
                }
                __syncwarp();
            }
            tc_fence_before();                                             // the output has been read: the next tile may overwrite it
            group_sync(2);                                                 // so have the exchanged numbers
            done_segment(k);
        }
        if (!fine && lane == 0 && p.status) atomicOr(p.status, kFlagCopyTimeout);
    }

    // ---- teardown: both blocks are done with each other's memory, and with tensor memory before it is released ----
    tc_fence_before();
    __syncthreads();
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
    if (warp == kPairWarpLogits) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" :: "r"(tmem), "n"(Geo::kTmemCols) : "memory");
    }
}

}  // namespace instinfer
