// Attention of draft trees on the fifth-generation tensor cores (tcgen05 MMAs, accumulators in tensor
// memory), head sizes 64, 128 and 256, for sm_100a.
//
// A tree puts up to 128 nodes times the heads of a group, R rows, against one KV head's cache: R
// flops per byte of K and V.  Up to about 260 rows the kernel is bound by HBM, as long as the exponentials
// (R per cached token) and the two contractions stay in its shadow.  So the QUERY ROWS are the long side of
// the MMAs here (the kernel for at most 16 rows has the tokens there):
//   S[128 rows x 128 tokens]  = Q[128 x D] K_tile^T           (both K-major, as they lie in memory)
//   O[128 rows x D]          += P[128 x 128] V_tile           (P from tensor memory, V MN-major)
// A row is a lane of tensor memory and belongs to one thread: its maximum, sum and rescaling need no
// exchange between threads.  The softmax weights go back to tensor memory over the logits they came
// from, each as an fp16 high and low part (P V is then two MMAs): the sum keeps the accuracy of 32-bit
// weights, where one fp16 part alone would add an error as large as the output's own rounding.
//
// Work split: the tiles of 128 tokens of all (sequence, KV head, row block) items lie in one row, and
// block c of G takes the tiles [W c / G, W (c + 1) / G) of the W there are, whatever
// items they belong to.  So every SM reads the same number of bytes, and only the items that a block
// starts or ends inside leave partial results: at most two per block (with fixed chunks the partials of
// a 16-sequence batch of 64 rows were 8 % of the traffic).  The cuts follow from the lengths alone,
// not from the placement of blocks.
//
// A block has 4 softmax warps per stream and four single-purpose warps, handing tiles over through mbarriers:
//   K producer, V producer   tensor-map copies into a ring each (128-byte swizzle); a paged tile is 128 / T
//                            copies of one (block, head) run; unreadable blocks are zero-filled;
//   logit and output issuer  one elected thread each issues the MMAs of S and of O.
// kStreams = 1 (at most 128 rows): two logit buffers, so that S of the next tile is computed while the
// softmax warps work on this one.  kStreams = 2: two row blocks share every K and V tile; each has its
// own softmax warps, logit buffer and accumulator, and the tensor cores serve them in turn.
// Every wait is bounded by the clock; one that runs out sets kFlagCopyTimeout, after which that warp
// waits no more, issues nothing more and ends.
#pragma once

#include "grouped_umma_kernels.cuh"
#include "tree_common.cuh"

namespace instinfer {

constexpr int kTreeTile = 128;                         // tokens per tile = rows per block of rows
constexpr int kTreePanelBytes = kTreeTile * 128;       // 64 dims of 128 rows
constexpr int kTreeMiscBytes = 1024;

template <int D, int kStreams>
struct TreeGeometry {
    static constexpr int kPanels = D / 64;
    static constexpr int kItemPanels = kPanels < 2 ? kPanels : 2;        // a ring item: up to 128 dims of a tile
    static constexpr int kItems = kPanels / kItemPanels;
    static constexpr int kItemBytes = kItemPanels * kTreePanelBytes;
    static constexpr int kItemDims = kItemPanels * 64;
    static constexpr int kQBytes = kPanels * kTreePanelBytes;            // per stream
    static constexpr int kRingItems = (224 * 1024 - kStreams * kQBytes) / kItemBytes;
    static constexpr int kKSlots = kRingItems / 2 < 6 ? kRingItems / 2 : 6;
    static constexpr int kVSlots = kRingItems - kKSlots < 6 ? kRingItems - kKSlots : 6;
    static constexpr int kRingBytes = (kKSlots + kVSlots) * kItemBytes;
    static constexpr int kCarveBytes = kRingBytes + kStreams * kQBytes + kTreeMiscBytes;
    static constexpr int kSmemBytes = kCarveBytes + 1024;                // room to align to 1024 bytes
    static constexpr int kSoftmaxWarps = 4 * kStreams;
    static constexpr int kThreads = (kSoftmaxWarps + 4) * 32;
    static constexpr int kOColumn = 256;                                 // tensor memory: two logit buffers, then the accumulators
    static_assert(kOColumn + kStreams * D <= 512, "tensor memory");
    static_assert(kKSlots >= kItems && kVSlots >= kItems, "a whole tile has to fit each ring");
    static_assert(kSmemBytes <= 227 * 1024, "one block per SM must fit");
};

// Offsets inside the misc region.
constexpr int kTreeBarKFull = 0;       // [6]
constexpr int kTreeBarKEmpty = 48;     // [6]
constexpr int kTreeBarVFull = 96;      // [6]
constexpr int kTreeBarVEmpty = 144;    // [6]
constexpr int kTreeBarSFull = 192;     // [2] logits of a unit are in tensor memory
constexpr int kTreeBarPFull = 208;     // [2] its weights are (4 warps)
constexpr int kTreeBarPvDone = 224;    // [2] its output MMAs are complete: the buffer is free, the accumulator is up to date
constexpr int kTreeBarQFull = 240;
constexpr int kTreeBarQEmpty = 248;
constexpr int kTreeTmemPtr = 256;
constexpr int kTreePoison = 272;       // [2][4] words: value rows of a tile that are not finite, by the parity of masked tiles
constexpr int kTreeStart = 304;        // where the block's tiles begin: sequence, tile inside it (64 bits), number of tiles
constexpr int kTreeScan = 384;         // [16] int64: per-warp sums of the set-up's scan
static_assert(kTreeScan + 16 * 8 <= kTreeMiscBytes, "misc region too small");

struct TreeParams {
    AttnParams a;              // heads = KV heads; part_o [2 G, rows, D], part_lse [2 G, rows]
    TreeShape tree;
    int32_t batch;
    int32_t group;             // query heads per KV head
    int32_t nodes_per_block;   // a row block is this many nodes' heads: row t * group + g of the block
    int32_t row_blocks;        // items per (sequence, KV head), kStreams row blocks each
    int32_t item_rows;         // kStreams * nodes_per_block * group
};

// Number of tiles of a sequence's items.
__device__ __forceinline__ int tree_tiles(int len, int nodes)
{
    return nodes > 0 ? (int)(((unsigned)len + kTreeTile - 1) / kTreeTile) : 0;
}

// The tile at which block `c` of `blocks` starts; blocks beyond the number of tiles have none.
__device__ __forceinline__ int64_t tree_first_tile(int64_t total, int c, int blocks)
{
    const int64_t working = min((int64_t)blocks, total);
    return c < working ? total * c / working : total;
}

// Tiles [t0, t1) of the n_tiles of one item.
struct TreeSegment {
    int b, len, nodes, hk, rb, t0, t1, n_tiles;
    __device__ __forceinline__ bool whole() const { return t0 == 0 && t1 == n_tiles; }
    __device__ __forceinline__ int prefix() const { return len - nodes; }
};

// The segments of one block, in order; every warp walks them by itself (all 32 lanes together).
struct TreeWalk {
    int b, len, nodes, item, tile;
    int64_t left;
    __device__ __forceinline__ void find(const TreeParams &p, int from, int lane)
    {
        // the next sequence from `from` on that has tiles (there is one as long as `left` is not 0)
        for (b = from; b < p.batch; b += 32) {
            int n = 0, l = 0;
            if (b + lane < p.batch) l = checked_tree(p.tree, p.a.seq_lens, p.a.max_seq_len, nullptr, b + lane, false, n);
            const unsigned live = __ballot_sync(0xffffffffu, tree_tiles(l, n) > 0);
            if (live == 0) continue;
            const int first = __ffs(live) - 1;
            b += first;
            len = __shfl_sync(0xffffffffu, l, first);
            nodes = __shfl_sync(0xffffffffu, n, first);
            return;
        }
        left = 0;
    }
    __device__ __forceinline__ void start(const TreeParams &p, const unsigned char *misc, int lane)
    {
        const int *at = reinterpret_cast<const int *>(misc + kTreeStart);
        const int64_t inside = *reinterpret_cast<const int64_t *>(misc + kTreeStart + 8);
        left = *reinterpret_cast<const int64_t *>(misc + kTreeStart + 16);
        find(p, at[0], lane);
        const int n = tree_tiles(len, nodes);
        item = n > 0 ? (int)(inside / n) : 0;
        tile = n > 0 ? (int)(inside - (int64_t)item * n) : 0;
    }
    __device__ __forceinline__ bool next(const TreeParams &p, TreeSegment &s, int lane)
    {
        if (left > 0 && item == p.a.heads * p.row_blocks) {
            find(p, b + 1, lane);
            item = 0;
            tile = 0;
        }
        if (left <= 0) return false;
        s.b = b;
        s.len = len;
        s.nodes = nodes;
        s.hk = item / p.row_blocks;
        s.rb = item - s.hk * p.row_blocks;
        s.n_tiles = tree_tiles(len, nodes);
        s.t0 = tile;
        s.t1 = (int)min((int64_t)s.n_tiles, tile + left);
        left -= s.t1 - s.t0;
        tile = s.t1;
        if (tile == s.n_tiles) {
            tile = 0;
            ++item;
        }
        return true;
    }
};

// ---- tensor-memory accesses of 32 columns ----
__device__ __forceinline__ void tc_issue_load32(float (&v)[32], unsigned taddr)      // valid after tc_loaded32
{
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 "
                 "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
                 "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
                 : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]), "=f"(v[4]), "=f"(v[5]), "=f"(v[6]), "=f"(v[7]),
                   "=f"(v[8]), "=f"(v[9]), "=f"(v[10]), "=f"(v[11]), "=f"(v[12]), "=f"(v[13]), "=f"(v[14]), "=f"(v[15]),
                   "=f"(v[16]), "=f"(v[17]), "=f"(v[18]), "=f"(v[19]), "=f"(v[20]), "=f"(v[21]), "=f"(v[22]), "=f"(v[23]),
                   "=f"(v[24]), "=f"(v[25]), "=f"(v[26]), "=f"(v[27]), "=f"(v[28]), "=f"(v[29]), "=f"(v[30]), "=f"(v[31])
                 : "r"(taddr) : "memory");
}
// Waits for this thread's loads; the values pass through, so that nothing uses them earlier.
__device__ __forceinline__ void tc_loaded32(float (&v)[32])
{
    asm volatile("tcgen05.wait::ld.sync.aligned;"
                 : "+f"(v[0]), "+f"(v[1]), "+f"(v[2]), "+f"(v[3]), "+f"(v[4]), "+f"(v[5]), "+f"(v[6]), "+f"(v[7]),
                   "+f"(v[8]), "+f"(v[9]), "+f"(v[10]), "+f"(v[11]), "+f"(v[12]), "+f"(v[13]), "+f"(v[14]), "+f"(v[15]),
                   "+f"(v[16]), "+f"(v[17]), "+f"(v[18]), "+f"(v[19]), "+f"(v[20]), "+f"(v[21]), "+f"(v[22]), "+f"(v[23]),
                   "+f"(v[24]), "+f"(v[25]), "+f"(v[26]), "+f"(v[27]), "+f"(v[28]), "+f"(v[29]), "+f"(v[30]), "+f"(v[31])
                 :: "memory");
}
__device__ __forceinline__ void tc_store32(unsigned taddr, const unsigned (&v)[32])  // complete after tc_stored
{
    asm volatile("tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], "
                 "{%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, "
                 "%17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31, %32};"
                 :: "r"(taddr), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]),
                    "r"(v[8]), "r"(v[9]), "r"(v[10]), "r"(v[11]), "r"(v[12]), "r"(v[13]), "r"(v[14]), "r"(v[15]),
                    "r"(v[16]), "r"(v[17]), "r"(v[18]), "r"(v[19]), "r"(v[20]), "r"(v[21]), "r"(v[22]), "r"(v[23]),
                    "r"(v[24]), "r"(v[25]), "r"(v[26]), "r"(v[27]), "r"(v[28]), "r"(v[29]), "r"(v[30]), "r"(v[31]) : "memory");
}
__device__ __forceinline__ void tc_stored() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
// D[tmem] (+)= A[tmem] B[smem]
__device__ __forceinline__ void tc_mma_f16_ts(unsigned d_tmem, unsigned a_tmem, uint64_t b_desc, unsigned idesc, unsigned accumulate)
{
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
                 "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
                 :: "r"(d_tmem), "r"(a_tmem), "l"(b_desc), "r"(idesc), "r"(accumulate) : "memory");
}

// 128 bits: what a row sees of a tile, one word per 32 tokens.
struct Bits128 {
    uint64_t lo, hi;
    __device__ __forceinline__ Bits128 shifted_up(int n) const           // 0 <= n < 128
    {
        if (n == 0) return *this;
        if (n >= 64) return {0, lo << (n - 64)};
        return {lo << n, hi << n | lo >> (64 - n)};
    }
    __device__ __forceinline__ Bits128 shifted_down(int n) const
    {
        if (n == 0) return *this;
        if (n >= 64) return {hi >> (n - 64), 0};
        return {lo >> n | hi << (64 - n), hi >> n};
    }
    __device__ __forceinline__ unsigned word(int i) const { return (unsigned)((i < 2 ? lo : hi) >> (32 * (i & 1))); }
};

template <int D, bool kPaged, int kStreams>
__global__ void __launch_bounds__(TreeGeometry<D, kStreams>::kThreads, 1)
tree_attn_umma_kernel(const TreeParams p, const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_k,
                      const __grid_constant__ CUtensorMap map_v)
{
    using Geo = TreeGeometry<D, kStreams>;
    constexpr int kItems = Geo::kItems, kItemPanels = Geo::kItemPanels, kItemBytes = Geo::kItemBytes;
    constexpr int kKSlots = Geo::kKSlots, kVSlots = Geo::kVSlots, kThreadsHere = Geo::kThreads;
    constexpr int kWarpK = Geo::kSoftmaxWarps, kWarpV = kWarpK + 1, kWarpLogits = kWarpK + 2, kWarpOutput = kWarpK + 3;
    extern __shared__ unsigned char smem_raw[];
    const AttnParams &a = p.a;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    allow_next_kernel();
    wait_for_previous_kernels();

    const unsigned raw = static_cast<unsigned>(__cvta_generic_to_shared(smem_raw));
    const unsigned base = (raw + 1023u) & ~1023u;
    unsigned char *smem = smem_raw + (base - raw);
    constexpr int kKOffset = 0, kVOffset = kKSlots * kItemBytes, kQOffset = Geo::kRingBytes;
    constexpr int kMiscOffset = kQOffset + kStreams * Geo::kQBytes;
    const unsigned q_smem = base + kQOffset, misc = base + kMiscOffset;
    unsigned char *misc_ptr = smem + kMiscOffset;

    // ---- set-up: where this block's tiles begin ----
    {
        const int per_thread = (p.batch + kThreadsHere - 1) / kThreadsHere;
        const int b0 = min((int)threadIdx.x * per_thread, p.batch), b1 = min(b0 + per_thread, p.batch);
        const int items = a.heads * p.row_blocks;
        int64_t mine = 0;
        for (int b = b0; b < b1; ++b) {
            int nodes;
            const int len = checked_tree(p.tree, a.seq_lens, a.max_seq_len, a.status, b, blockIdx.x == 0, nodes);
            mine += (int64_t)tree_tiles(len, nodes) * items;
        }
        int64_t run = mine;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int64_t up = __shfl_up_sync(0xffffffffu, run, o);
            if (lane >= o) run += up;
        }
        int64_t *scan = reinterpret_cast<int64_t *>(misc_ptr + kTreeScan);
        if (lane == 31) scan[warp] = run;
        if (threadIdx.x == 0) {                        // no tiles, unless a thread finds the first one below
            *reinterpret_cast<int *>(misc_ptr + kTreeStart) = 0;
            *reinterpret_cast<int64_t *>(misc_ptr + kTreeStart + 8) = 0;
            *reinterpret_cast<int64_t *>(misc_ptr + kTreeStart + 16) = 0;
        }
        __syncthreads();
        int64_t before = 0, total = 0;
        for (int w = 0; w < kThreadsHere / 32; ++w) {
            if (w < warp) before += scan[w];
            total += scan[w];
        }
        const int64_t first = tree_first_tile(total, blockIdx.x, gridDim.x), last = tree_first_tile(total, blockIdx.x + 1, gridDim.x);
        int64_t at = before + run - mine;
        if (first < last && at <= first && first < at + mine) {
            for (int b = b0; b < b1; ++b) {
                int nodes;
                const int len = checked_tree(p.tree, a.seq_lens, a.max_seq_len, nullptr, b, false, nodes);
                const int64_t n = (int64_t)tree_tiles(len, nodes) * items;
                if (first < at + n) {
                    *reinterpret_cast<int *>(misc_ptr + kTreeStart) = b;
                    *reinterpret_cast<int64_t *>(misc_ptr + kTreeStart + 8) = first - at;
                    *reinterpret_cast<int64_t *>(misc_ptr + kTreeStart + 16) = last - first;
                    break;
                }
                at += n;
            }
        }
    }
    if (warp == kWarpLogits) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;"
                     :: "r"(misc + kTreeTmemPtr), "n"(512) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    } else if (warp == kWarpK) {
        if (lane == 0) {
#pragma unroll
            for (int s = 0; s < 6; ++s) {
                mbarrier_init(misc + kTreeBarKFull + s * 8, 1);
                mbarrier_init(misc + kTreeBarKEmpty + s * 8, 1);
                mbarrier_init(misc + kTreeBarVFull + s * 8, 1);
                mbarrier_init(misc + kTreeBarVEmpty + s * 8, 1);
            }
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                mbarrier_init(misc + kTreeBarSFull + s * 8, 1);
                mbarrier_init(misc + kTreeBarPFull + s * 8, 4);
                mbarrier_init(misc + kTreeBarPvDone + s * 8, 1);
            }
            mbarrier_init(misc + kTreeBarQFull, 1);
            mbarrier_init(misc + kTreeBarQEmpty, 1);
            mbarrier_init_fence();
            asm volatile("prefetch.tensormap [%0];" :: "l"(reinterpret_cast<uint64_t>(&map_q)) : "memory");
            asm volatile("prefetch.tensormap [%0];" :: "l"(reinterpret_cast<uint64_t>(&map_k)) : "memory");
            asm volatile("prefetch.tensormap [%0];" :: "l"(reinterpret_cast<uint64_t>(&map_v)) : "memory");
        }
    } else if (warp < Geo::kSoftmaxWarps) {
        // rows of a block that do not exist are zeros for good: the copies fill only the others
        const uint4 zero = make_uint4(0u, 0u, 0u, 0u);
        for (int i = threadIdx.x; i < kStreams * Geo::kQBytes / 16; i += Geo::kSoftmaxWarps * 32)
            *reinterpret_cast<uint4 *>(smem + kQOffset + i * 16) = zero;
        fence_async_proxy();
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const unsigned tmem = *reinterpret_cast<volatile unsigned *>(misc_ptr + kTreeTmemPtr);
    TreeWalk walk;
    walk.start(p, misc_ptr, lane);
    TreeSegment seg;

    // The buffer of a unit (tile number g of this block, stream s) and how often it was used before.
    auto buffer_of = [](int g, int s) -> int { return kStreams == 1 ? g & 1 : s; };
    auto use_of = [](int g) -> int { return kStreams == 1 ? g >> 1 : g; };

    // One tile of one cache into its ring (all lanes); `ids`: lane i's physical block for the tile.
    const int T = kPaged ? min(a.block_tokens, kTreeTile) : kTreeTile;
    auto fetch_ids = [&](const TreeSegment &s, int j) -> int {
        if (!kPaged) return 0;
        const int start = j * kTreeTile;
        if (j >= s.t1 || lane >= (min(s.len - start, kTreeTile) + T - 1) / T) return -1;
        const int idx = (start + lane * T) / a.block_tokens;
        return bounds_ok(idx < a.max_blocks_per_seq, a.status) ? __ldg(a.block_table + (int64_t)s.b * a.max_blocks_per_seq + idx) : -1;
    };
    auto copy_tile = [&](const TreeSegment &s, int j, int phys, const CUtensorMap *map, int ring_offset, int slots, int bar_full,
                         int bar_empty, int &count) -> bool {
        const int start = j * kTreeTile;
        const int nb = kPaged ? (min(s.len - start, kTreeTile) + T - 1) / T : 1;
        bool good = lane < nb;
        int row0;
        if (kPaged) {
            const bool in_range = phys >= 0 && (int64_t)phys < a.num_phys_blocks;
            if (good && !in_range && a.status) atomicOr(a.status, kFlagBlockRange);
            // (< 2^31 rows: checked by the host)
            row0 = in_range ? (phys * a.heads + s.hk) * a.block_tokens + (start + lane * T) % a.block_tokens : 0;
            good = good && in_range && bounds_ok((int64_t)row0 + T <= a.kv_bytes / (2 * D), a.status);
        } else {
            row0 = (s.b * a.heads + s.hk) * a.s_max + start;      // rows past the tensor's end read as zeros
        }
        const unsigned fetched = __popc(__ballot_sync(0xffffffffu, good));
#pragma unroll
        for (int item = 0; item < kItems; ++item, ++count) {
            const int slot = count % slots;
            if (count >= slots &&
                !__all_sync(0xffffffffu, mbarrier_wait_bounded(misc + bar_empty + slot * 8, (count / slots - 1) & 1)))
                return false;
            const int slot_offset = ring_offset + slot * kItemBytes + (kPaged ? lane * T * 128 : 0);
            const unsigned bar = misc + bar_full + slot * 8;
            if (kPaged && lane < nb && !good) {                   // a block that cannot be read counts as zeros
                const uint4 zero = make_uint4(0u, 0u, 0u, 0u);
                for (int i = 0; i < T * 8; ++i) {
#pragma unroll
                    for (int panel = 0; panel < kItemPanels; ++panel)
                        *reinterpret_cast<uint4 *>(smem + slot_offset + panel * kTreePanelBytes + i * 16) = zero;
                }
                fence_async_proxy();
            }
            if (lane == 0) mbarrier_expect_bytes(bar, fetched * (unsigned)(T * 128 * kItemPanels));
            __syncwarp();
            if (good) {
#pragma unroll
                for (int panel = 0; panel < kItemPanels; ++panel)
                    tma_load_2d(base + slot_offset + panel * kTreePanelBytes, map, (item * kItemPanels + panel) * 64, row0, bar);
            }
        }
        return true;
    };
    // copies in flight must land (or be given up, bounded) before shared memory is handed on
    auto drain = [&](int bar_full, int slots, int count) {
        for (int i = max(count - slots, 0); i < count; ++i)
            (void)mbarrier_poll_bounded(misc + bar_full + (i % slots) * 8, (i / slots) & 1);
    };

    if (warp == kWarpK) {
        // ================================ K producer, and the query rows ================================
        int count = 0, k = 0;
        bool fine = true;
        for (; fine && walk.next(p, seg, lane); ++k) {
            int ids = fetch_ids(seg, seg.t0);
            for (int j = seg.t0; j < seg.t1 && fine; ++j) {
                const int now = ids;
                ids = fetch_ids(seg, j + 1);
                fine = copy_tile(seg, j, now, &map_k, kKOffset, kKSlots, kTreeBarKFull, kTreeBarKEmpty, count);
                if (j > seg.t0 || !fine) continue;
                // the item's query rows, behind its first K tile: they wait for the last item's logits
                if (k >= 1) fine = __all_sync(0xffffffffu, mbarrier_wait_bounded(misc + kTreeBarQEmpty, (k - 1) & 1));
                if (fine && lane == 0) {
                    const int rows_bytes = p.nodes_per_block * p.group * 128;
                    int blocks = 0;
#pragma unroll
                    for (int s = 0; s < kStreams; ++s) blocks += (seg.rb * kStreams + s) * p.nodes_per_block < p.tree.tokens;
                    mbarrier_expect_bytes(misc + kTreeBarQFull, (unsigned)(blocks * rows_bytes * Geo::kPanels));
#pragma unroll
                    for (int s = 0; s < kStreams; ++s) {
                        const int node0 = (seg.rb * kStreams + s) * p.nodes_per_block;
                        if (node0 >= p.tree.tokens) continue;
#pragma unroll
                        for (int panel = 0; panel < Geo::kPanels; ++panel)
                            tma_load_4d(q_smem + s * Geo::kQBytes + panel * kTreePanelBytes, &map_q, panel * 64, seg.hk * p.group,
                                        node0, seg.b, misc + kTreeBarQFull);
                    }
                }
                __syncwarp();
            }
        }
        if (!fine) {
            if (lane == 0 && a.status) atomicOr(a.status, kFlagCopyTimeout);
            drain(kTreeBarKFull, kKSlots, count);
            if (k >= 1) (void)mbarrier_poll_bounded(misc + kTreeBarQFull, (k - 1) & 1);
        }
    } else if (warp == kWarpV) {
        // ================================ V producer ================================
        int count = 0;
        bool fine = true;
        while (fine && walk.next(p, seg, lane)) {
            int ids = fetch_ids(seg, seg.t0);
            for (int j = seg.t0; j < seg.t1 && fine; ++j) {
                const int now = ids;
                ids = fetch_ids(seg, j + 1);
                fine = copy_tile(seg, j, now, &map_v, kVOffset, kVSlots, kTreeBarVFull, kTreeBarVEmpty, count);
            }
        }
        if (!fine) {
            if (lane == 0 && a.status) atomicOr(a.status, kFlagCopyTimeout);
            drain(kTreeBarVFull, kVSlots, count);
        }
    } else if (warp == kWarpLogits) {
        // ================================ logit MMAs ================================
        constexpr unsigned idesc = umma_idesc(128, 128, 0, 0);
        bool fine = true;
        int g = 0;
        for (int k = 0; fine && walk.next(p, seg, lane); ++k) {
            fine = __all_sync(0xffffffffu, mbarrier_wait_bounded(misc + kTreeBarQFull, k & 1));
            for (int j = seg.t0; j < seg.t1 && fine; ++j, ++g) {
#pragma unroll
                for (int item = 0; item < kItems; ++item) {
                    if (!fine) break;
                    const int n = g * kItems + item, slot = n % kKSlots;
                    fine = __all_sync(0xffffffffu, mbarrier_wait_bounded(misc + kTreeBarKFull + slot * 8, (n / kKSlots) & 1));
                    if (!fine) break;
                    // rows of 128 bytes per 64-dim panel, 8-row groups 1024 bytes apart; a k-step of 16
                    // dims is 32 bytes along the row
                    const uint64_t k_desc = umma_desc(base + kKOffset + slot * kItemBytes, 16, 1024, 2);
#pragma unroll
                    for (int s = 0; s < kStreams; ++s) {
                        const int buf = buffer_of(g, s), use = use_of(g);
                        if (item == 0 && use >= 1)             // the weights that lie in the buffer have been used
                            fine = fine && __all_sync(0xffffffffu, mbarrier_wait_bounded(misc + kTreeBarPvDone + buf * 8, (use - 1) & 1));
                        if (!fine) break;
                        tc_fence_after();
                        const uint64_t q_desc = umma_desc(q_smem + s * Geo::kQBytes, 16, 1024, 2);
                        if (elect_one()) {
#pragma unroll
                            for (int ks = 0; ks < 4 * kItemPanels; ++ks)
                                tc_mma_f16(tmem + buf * 128,
                                           q_desc + (uint64_t)(((item * kItemPanels + (ks >> 2)) * kTreePanelBytes + (ks & 3) * 32) >> 4),
                                           k_desc + (uint64_t)(((ks >> 2) * kTreePanelBytes + (ks & 3) * 32) >> 4), idesc,
                                           item > 0 || ks > 0);
                            if (item + 1 == kItems) tc_commit(misc + kTreeBarSFull + buf * 8);
                            if (s + 1 == kStreams) {
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
        constexpr unsigned idesc = umma_idesc(128, Geo::kItemDims, 0, 1);         // weights K-major, V MN-major
        bool fine = true;
        int g = 0;
        while (fine && walk.next(p, seg, lane)) {
            for (int j = seg.t0; j < seg.t1 && fine; ++j, ++g) {
#pragma unroll
                for (int s = 0; s < kStreams; ++s) {
                    const int buf = buffer_of(g, s);
                    fine = fine && __all_sync(0xffffffffu, mbarrier_poll_bounded(misc + kTreeBarPFull + buf * 8, use_of(g) & 1));
#pragma unroll
                    for (int item = 0; item < kItems; ++item) {
                        const int n = g * kItems + item, slot = n % kVSlots;
                        if (s == 0 && fine)
                            fine = __all_sync(0xffffffffu, mbarrier_poll_bounded(misc + kTreeBarVFull + slot * 8, (n / kVSlots) & 1));
                        if (!fine) break;
                        tc_fence_after();
                        // 64-dim panels kTreePanelBytes apart, 8-token groups 1024 bytes apart; a k-step is
                        // 16 tokens = 2048 bytes.  Weights of 32 tokens: 16 columns of high, 16 of low parts.
                        const uint64_t v_desc = umma_desc(base + kVOffset + slot * kItemBytes, kTreePanelBytes, 1024, 2);
                        if (elect_one()) {
                            const unsigned acc = tmem + Geo::kOColumn + s * D + item * 128, weights = tmem + buf * 128;
#pragma unroll
                            for (int ks = 0; ks < 8; ++ks) {
                                const unsigned at = weights + (ks >> 1) * 32 + (ks & 1) * 8;
                                const uint64_t v_step = v_desc + (uint64_t)((ks * 2048) >> 4);
                                tc_mma_f16_ts(acc, at, v_step, idesc, j > seg.t0 || ks > 0);
                                tc_mma_f16_ts(acc, at + 16, v_step, idesc, 1);
                            }
                            if (s + 1 == kStreams) tc_commit(misc + kTreeBarVEmpty + slot * 8);
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
        volatile unsigned *poison_words = reinterpret_cast<volatile unsigned *>(misc_ptr + kTreePoison);
        bool fine = true;
        int g = 0, masked_tiles = 0;
        while (walk.next(p, seg, lane)) {
            const int node = (seg.rb * kStreams + s) * p.nodes_per_block + node_in_block;
            const bool exists = used_row && node < p.tree.tokens, live = exists && node < seg.nodes;
            const int prefix = seg.prefix();
            TreeRow row = {0, 0, live};
            if (live && seg.t1 * kTreeTile > prefix) row = tree_row(p.tree, seg.b, node, seg.nodes);
            Bits128 poison = {0, 0};                                  // nodes whose value row was taken out of a tile
            float m = kMinusHuge, l = 0.f;                            // l and the accumulator carry kGroupWeightScale
            for (int j = seg.t0; j < seg.t1; ++j, ++g) {
                const int buf = buffer_of(g, s), start = j * kTreeTile;
                const unsigned logits = tmem + lanes + buf * 128;
                const bool masked = start + kTreeTile > prefix;       // uniform
                if (masked) {
                    // Value rows behind the sequence get weight 0 but may hold anything, and 0 x NaN is NaN:
                    // they are cleared.  A node's row that is not finite is cleared too, and added at the end
                    // for the rows that see it.  kStreams threads look through one row.
                    const int row_here = (int)threadIdx.x / kStreams, part = (int)threadIdx.x % kStreams;
                    const int pos = start + row_here;
                    const bool look = pos >= prefix;
                    bool bad = false;
                    uint4 *rows[kItems];
#pragma unroll
                    for (int item = 0; item < kItems; ++item) {
                        const int n = g * kItems + item, slot = n % kVSlots;
                        if (fine) fine = mbarrier_poll_bounded(misc + kTreeBarVFull + slot * 8, (n / kVSlots) & 1);
                        rows[item] = reinterpret_cast<uint4 *>(smem + kVOffset + slot * kItemBytes + row_here * 128);
                    }
                    __syncwarp();
                    // 16-byte piece i of the row: panels of 8 pieces
                    auto piece = [&](int i) -> uint4 & {
                        return rows[i / (8 * kItemPanels)][(i / 8) % kItemPanels * (kTreePanelBytes / 16) + i % 8];
                    };
                    if (look && pos < seg.len) {
#pragma unroll
                        for (int i = 0; i < Geo::kPanels * 8; i += kStreams) bad = bad || !finite8(piece(i + part));
                    }
                    __syncwarp();
                    if (kStreams == 2) bad = __shfl_xor_sync(0xffffffffu, (int)bad, 1) || bad;
                    if (bad || (look && pos >= seg.len)) {
#pragma unroll
                        for (int i = 0; i < Geo::kPanels * 8; i += kStreams) piece(i + part) = make_uint4(0u, 0u, 0u, 0u);
                        fence_async_proxy();
                    }
                    __syncwarp();
                    const unsigned ballot = __ballot_sync(0xffffffffu, bad);
                    volatile unsigned *words = poison_words + (masked_tiles & 1) * 4;
                    if (kStreams == 1) {
                        if (lane == 0) words[warp] = ballot;
                    } else {                                          // two lanes per row: 16 rows a warp
                        unsigned half = 0;
                        for (int i = 0; i < 16; ++i) half |= (ballot >> (2 * i) & 1u) << i;
                        if (lane == 0) reinterpret_cast<volatile unsigned short *>(words)[warp] = (unsigned short)half;
                    }
                    asm volatile("bar.sync 1, %0;" :: "n"(128 * kStreams) : "memory");
                    Bits128 found = {words[0] | (uint64_t)words[1] << 32, words[2] | (uint64_t)words[3] << 32};
                    ++masked_tiles;
                    if (found.lo | found.hi) {
                        found = start < prefix ? found.shifted_down(prefix - start) : found.shifted_up(start - prefix);
                        poison.lo |= found.lo;
                        poison.hi |= found.hi;
                    }
                }
                if (fine) fine = mbarrier_poll_bounded(misc + kTreeBarSFull + buf * 8, use_of(g) & 1);
                fine = __all_sync(0xffffffffu, fine);
                tc_fence_after();
                float x[4][32];
#pragma unroll
                for (int i = 0; i < 4; ++i) tc_issue_load32(x[i], logits + i * 32);
#pragma unroll
                for (int i = 0; i < 4; ++i) tc_loaded32(x[i]);
                float factor = a.scale_log2e;
                if (masked || factor < 0.f) {                         // uniform; a negative scale would turn the maximum around
                    Bits128 sees = {~(uint64_t)0, ~(uint64_t)0};
                    if (masked) {
                        sees = {row.lo, row.hi};
                        if (start < prefix) {
                            const int n = prefix - start;             // 1 .. 127 tokens before the tree
                            sees = sees.shifted_up(n);
                            if (row.all) {
                                sees.lo |= n >= 64 ? ~(uint64_t)0 : ((uint64_t)1 << n) - 1;
                                if (n > 64) sees.hi |= ((uint64_t)1 << (n - 64)) - 1;
                            }
                        } else {
                            sees = sees.shifted_down(start - prefix);
                        }
                    }
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const unsigned word = sees.word(i);
#pragma unroll
                        for (int c = 0; c < 32; ++c) x[i][c] = word >> c & 1u ? x[i][c] * factor : -INFINITY;
                    }
                    factor = 1.f;
                }
                float top4[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    top4[i] = x[i][0];
#pragma unroll
                    for (int c = 1; c < 32; ++c) top4[i] = fmaxf(top4[i], x[i][c]);
                }
                const float top = fmaxf(fmaxf(top4[0], top4[1]), fmaxf(top4[2], top4[3])) * factor;
                // The reference follows the maximum lazily: weights stay below 2^kGroupLag.
                const bool moved = top > m + kGroupLag;
                if (__any_sync(0xffffffffu, moved)) {
                    const float alpha = moved ? fast_exp2(m - top) : 1.f;
                    if (moved) m = top;
                    l *= alpha;
                    if (j > seg.t0) {
                        // the accumulator holds the tiles before this one once their MMAs are complete
                        if (fine) fine = mbarrier_poll_bounded(misc + kTreeBarPvDone + buffer_of(g - 1, s) * 8, use_of(g - 1) & 1);
                        fine = __all_sync(0xffffffffu, fine);
                        tc_fence_after();
#pragma unroll
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
                const float ref = m - kGroupWeightLog2;
                float sums[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    unsigned parts[32];
#pragma unroll
                    for (int c = 0; c < 16; ++c) {
                        const float w0 = fast_exp2(fmaf(x[i][2 * c], factor, -ref)), w1 = fast_exp2(fmaf(x[i][2 * c + 1], factor, -ref));
                        sums[c & 1] += w0;
                        sums[2 + (c & 1)] += w1;
                        parts[c] = pack_half2(w0, w1);
                        const float2 back = __half22float2(*reinterpret_cast<const __half2 *>(&parts[c]));
                        parts[16 + c] = pack_half2(w0 - back.x, w1 - back.y);
                    }
                    tc_store32(logits + i * 32, parts);
                }
                l += (sums[0] + sums[1]) + (sums[2] + sums[3]);
                tc_stored();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbarrier_arrive(misc + kTreeBarPFull + buf * 8);
            }
            // ---- the segment's end: the accumulator divided by the sum, to the output or the workspace ----
            if (fine) fine = mbarrier_poll_bounded(misc + kTreeBarPvDone + buffer_of(g - 1, s) * 8, use_of(g - 1) & 1);
            fine = __all_sync(0xffffffffu, fine);
            tc_fence_after();
            const bool empty = !live || l == 0.f;                     // (a NaN sum is not an empty row's)
            const float inverse = empty ? 0.f : 1.f / l;
            const float lse2 = empty ? kMinusHuge : m + log2f(l) - kGroupWeightLog2;
            const int64_t out_row = ((int64_t)seg.b * p.tree.tokens + node) * ((int64_t)a.heads * p.group) + (int64_t)seg.hk * p.group + head;
            // the rows that a block starts inside go to its first slot, those it ends inside to its second
            const int64_t slot_row = (int64_t)(2 * blockIdx.x + (seg.t0 == 0 ? 1 : 0)) * p.item_rows + s * p.nodes_per_block * p.group + t;
            const bool whole = seg.whole();
            const bool stray = ((poison.lo & row.lo) | (poison.hi & row.hi)) != 0;
#pragma unroll
            for (int c0 = 0; c0 < D; c0 += 32) {
                float o[32];
                tc_issue_load32(o, acc + c0);
                tc_loaded32(o);
                if (exists && fine) {
#pragma unroll
                    for (int c = 0; c < 32; ++c) o[c] = empty ? 0.f : o[c] * inverse;
                    if (stray) {                                          // rare: value rows with infinities or NaN that this row sees
                        for (int n = 0; n < seg.nodes; ++n) {
                            if (!((n < 64 ? poison.lo : poison.hi) >> (n & 63) & 1u) || !row.sees(n)) continue;
                            const int64_t kv_row = tree_cache_row(a, seg.b, seg.hk, prefix + n);
                            float dot = 0.f;
                            for (int c = 0; c < D; ++c) dot = fmaf(__half2float(a.q[out_row * D + c]), __half2float(a.k[kv_row * D + c]), dot);
                            const float weight = fast_exp2(dot * a.scale_log2e - lse2);
#pragma unroll
                            for (int c = 0; c < 32; ++c) o[c] += weight * __half2float(a.v[kv_row * D + c0 + c]);
                        }
                    }
                    if (whole) {
                        uint4 *to = reinterpret_cast<uint4 *>(a.out + out_row * D + c0);
#pragma unroll
                        for (int c = 0; c < 32; c += 8)
                            to[c / 8] = make_uint4(pack_half2(o[c], o[c + 1]), pack_half2(o[c + 2], o[c + 3]),
                                                   pack_half2(o[c + 4], o[c + 5]), pack_half2(o[c + 6], o[c + 7]));
                    } else {
                        float4 *to = reinterpret_cast<float4 *>(a.part_o + slot_row * D + c0);
#pragma unroll
                        for (int c = 0; c < 32; c += 4) to[c / 4] = make_float4(o[c], o[c + 1], o[c + 2], o[c + 3]);
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

// Joins the partial results of the items that more than one block worked on, and zeroes the rows of
// sequences without work; one thread block per item and kTreeMergeRows rows, one warp per row.
constexpr int kTreeMergeThreads = 128;
constexpr int kTreeMergeRows = 16;

template <int D>
__global__ void __launch_bounds__(kTreeMergeThreads)
tree_merge_kernel(const TreeParams p, int blocks, int row_parts)
{
    const AttnParams &a = p.a;
    __shared__ int64_t sums[2][kTreeMergeThreads / 32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int part = blockIdx.x % row_parts;
    const int item = blockIdx.x / row_parts;                          // (sequence, KV head, row block)
    const int items = a.heads * p.row_blocks;
    const int b = item / items, in_seq = item - b * items;
    const int hk = in_seq / p.row_blocks, rb = in_seq - hk * p.row_blocks;
    allow_next_kernel();
    wait_for_previous_kernels();
    int nodes;
    const int len = checked_tree(p.tree, a.seq_lens, a.max_seq_len, nullptr, b, false, nodes);
    const int n_tiles = tree_tiles(len, nodes);
    int c0 = 0, c1 = 0;
    if (n_tiles > 0) {
        // tiles before this sequence, and all of them
        int64_t before = 0, all = 0;
        for (int i = threadIdx.x; i < p.batch; i += kTreeMergeThreads) {
            int n;
            const int other = checked_tree(p.tree, a.seq_lens, a.max_seq_len, nullptr, i, false, n);
            const int64_t tiles = (int64_t)tree_tiles(other, n) * items;
            if (i < b) before += tiles;
            all += tiles;
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) {
            before += __shfl_xor_sync(0xffffffffu, before, o);
            all += __shfl_xor_sync(0xffffffffu, all, o);
        }
        if (lane == 0) {
            sums[0][warp] = before;
            sums[1][warp] = all;
        }
        __syncthreads();
        before = all = 0;
        for (int w = 0; w < kTreeMergeThreads / 32; ++w) {
            before += sums[0][w];
            all += sums[1][w];
        }
        const int64_t first = before + (int64_t)in_seq * n_tiles, last = first + n_tiles - 1;
        auto block_of = [&](int64_t tile) -> int {
            int c = (int)(tile * min((int64_t)blocks, all) / all);
            while (tree_first_tile(all, c + 1, blocks) <= tile) ++c;
            while (tree_first_tile(all, c, blocks) > tile) --c;
            return c;
        };
        c0 = block_of(first);
        c1 = block_of(last);
        if (c0 == c1) return;                                         // one block had it all: the result is written
    }
    constexpr int kPer = D / 32;                                      // dims per lane
    for (int r = part * kTreeMergeRows + warp; r < min((part + 1) * kTreeMergeRows, p.item_rows); r += kTreeMergeThreads / 32) {
        const int node = rb * (p.item_rows / p.group) + r / p.group, head = r % p.group;
        if (node >= p.tree.tokens) continue;
        const int64_t out_row = ((int64_t)b * p.tree.tokens + node) * ((int64_t)a.heads * p.group) + (int64_t)hk * p.group + head;
        float top = kMinusHuge, total = 0.f, acc[kPer];
        bool any_nan = false;
#pragma unroll
        for (int i = 0; i < kPer; ++i) acc[i] = 0.f;
        auto slot_row = [&](int c) -> int64_t { return (int64_t)(2 * c + (c == c0 ? 1 : 0)) * p.item_rows + r; };
        if (n_tiles > 0) {
            for (int c = c0; c <= c1; ++c) {
                const float lse = a.part_lse[slot_row(c)];
                top = fmaxf(top, lse);
                any_nan = any_nan || lse != lse;
            }
            if (top > kMinusHuge || any_nan) {
                for (int c = c0; c <= c1; ++c) {
                    const float w = fast_exp2(a.part_lse[slot_row(c)] - top);
                    total += w;
                    const float *from = a.part_o + slot_row(c) * D + lane * kPer;
#pragma unroll
                    for (int i = 0; i < kPer; ++i) acc[i] = fmaf(w, from[i], acc[i]);
                }
            }
        }
        const bool empty = !(top > kMinusHuge) && !any_nan;
#pragma unroll
        for (int i = 0; i < kPer; ++i) a.out[out_row * D + lane * kPer + i] = __float2half_rn(empty ? 0.f : acc[i] / total);
        if (a.lse && lane == 0) a.lse[out_row] = empty ? -INFINITY : (top + log2f(total)) * kLn2;
    }
}

}  // namespace instinfer
