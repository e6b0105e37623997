// What the tcgen05 kernels for draft trees share (tree_umma_rows.cuh, tree_umma_tokens.cuh), for sm_100a: the
// split of the work, the walk through it, the copies, and the merge of partial results.
//
// Work split: the tiles of 128 tokens of all (sequence, KV head, row block) items lie in one row of W tiles,
// which is cut into pieces whatever items they belong to: first one long piece per block, 11/16 of the
// tiles together, then short ones that the blocks draw from a ticket counter.  Only the items that a
// piece starts or ends inside leave partial results, two per piece at most (with the fixed chunks of the
// other kernels the partials of 64 rows are 8 % of the traffic).  Why not equal shares alone: the SMs do not reach
// memory equally fast, with equal shares of 207 tiles the first was done after 312 us and the last after 399.
// (An item that is short next to the long pieces stays whole with the long piece that it starts in.)
// Few tiles are cut into equal shares, one per block.  A segment's set-up and end cost as much as some tiles, so an
// item counts that many more (in front of its first): a block full of short sequences gets fewer of
// them (104 -> 70 us at 35 items of 1 to 157 tiles).  The cuts follow from the lengths alone, so a result
// depends neither on which block draws a piece nor on the placement of the cache's blocks.
//
// A block has softmax warps and four single-purpose warps, which hand tiles over through mbarriers:
//   K producer               draws the pieces and announces their segments (a piece's part of one item) to the
//                            others through a queue in shared memory; copies K tiles and query rows;
//   V producer               the V tiles.  Both: tensor-map copies into a ring each (128-byte swizzle); a paged tile is 128 / T
//                            copies of one (block, head) run; unreadable blocks are zero-filled;
//   logit and output issuer  one elected thread each issues the MMAs of the logits and of the output.
// Every wait is bounded by the clock; one that runs out sets kFlagCopyTimeout, after which that warp
// waits no more, issues nothing more and ends.
#pragma once

#include "grouped_umma_kernels.cuh"
#include "tree_common.cuh"

namespace instinfer {

constexpr int kTreeTile = 128;                         // tokens per tile
constexpr int kTreePanelBytes = kTreeTile * 128;       // 64 dims of 128 rows

// A bounded wait with the loop out of line: the first test succeeds more often than not, and some thirty of these
// are in each kernel.  (Polling instead of the parked wait made no difference here.)
static __device__ __noinline__ bool tree_wait_more(unsigned bar, unsigned parity) { return mbarrier_wait_bounded(bar, parity); }
__device__ __forceinline__ bool tree_wait(unsigned bar, unsigned parity) { return mbarrier_test(bar, parity) || tree_wait_more(bar, parity); }

// Ring geometry of a head size: an item is up to 128 dims of a tile (32 KiB; 16 KiB at head size 64).
template <int D, int kBytes>
struct TreeRing {
    static constexpr int kPanels = D / 64;
    static constexpr int kItemPanels = kPanels < 2 ? kPanels : 2;
    static constexpr int kItems = kPanels / kItemPanels;                 // items per tile and cache
    static constexpr int kItemBytes = kItemPanels * kTreePanelBytes;
    static constexpr int kTotal = kBytes / kItemBytes;
    static constexpr int kKSlots = kTotal / 2 < 6 ? kTotal / 2 : 6;
    static constexpr int kVSlots = kTotal - kKSlots < 6 ? kTotal - kKSlots : 6;
    static constexpr int kVOffset = kKSlots * kItemBytes;
    static constexpr int kRingBytes = (kKSlots + kVSlots) * kItemBytes;
    static_assert(kKSlots >= kItems && kVSlots >= kItems, "a whole tile has to fit each ring");
};

// Offsets inside the misc region that the kernels have in common.
constexpr int kTreeBarKFull = 0;       // [6]
constexpr int kTreeBarKEmpty = 48;     // [6]
constexpr int kTreeBarVFull = 96;      // [6]
constexpr int kTreeBarVEmpty = 144;    // [6]
constexpr int kTreeBarSFull = 192;     // [4] logits of a unit are in tensor memory
constexpr int kTreeBarPFull = 224;     // [4] its weights are where the output MMAs read them
constexpr int kTreeBarPvDone = 256;    // [4] its output MMAs are complete
constexpr int kTreeBarQFull = 288;
constexpr int kTreeBarQEmpty = 296;
constexpr int kTreeBarSFree = 304;     // [2] the logits have been read
constexpr int kTreeTmemPtr = 320;
constexpr int kTreeTotal = 328;        // number of tiles
constexpr int kTreeBarSegFull = 336;   // [4] a segment is announced
constexpr int kTreeBarSegEmpty = 368;  // [4] everyone is done with it
constexpr int kTreePoison = 400;       // [8][4] words: nodes of a segment whose value row is not finite, by segment number
constexpr int kTreeSegments = 528;     // [4] TreeSegment
constexpr int kTreeEntryBytes = 56;
constexpr int kTreeScan = 528;         // [16] ints: per-warp sums of the set-up's scan, before the first segment
constexpr int kTreeMiscBytes = 528 + 4 * kTreeEntryBytes;
static_assert(kTreeScan + 16 * 4 <= kTreeMiscBytes && kTreeMiscBytes % 16 == 0, "misc region too small");

struct TreeParams {
    AttnParams a;              // heads = KV heads; part_o [2 G, item_rows, D], part_lse [2 G, item_rows]
    TreeShape tree;
    int32_t batch;
    int32_t group;             // query heads per KV head
    int32_t nodes_per_block;   // a row block is this many nodes' heads: row t * group + g of the block
    int32_t row_blocks;        // items per (sequence, KV head), of one or two row blocks each
    int32_t item_rows;         // rows of an item: all its row blocks'
    int32_t short_pieces;      // drawn pieces per block
    int2 *item_pieces;         // [items] the pieces with the item's first and its last tile, for the merge
    unsigned *ticket;          // zero before the launch where W can reach kTreeDrawnTiles per block
};

constexpr int kTreeItemCost = 4;

// Number of tiles of a sequence's items.
__device__ __forceinline__ int tree_tiles(int len, int nodes)
{
    return nodes > 0 ? (int)(((unsigned)len + kTreeTile - 1) / kTreeTile) : 0;
}

// What an item counts in the row of tiles.
__device__ __forceinline__ int tree_weight(int tiles) { return tiles > 0 ? tiles + kTreeItemCost : 0; }

// The cut of the row of tiles (see above); piece c is [first(c), first(c + 1)), count() pieces in all.
constexpr int kTreeDrawnTiles = 24;    // tiles per block from which on pieces are drawn
struct TreePieces {
    int total, length, drawn;          // W; tiles of a long piece; first tile of the short pieces
    int blocks, step;                  // step: tiles of a short piece, 0: none
    __device__ __forceinline__ TreePieces(int total_, int grid, int short_pieces)
        : total(total_), length(0), drawn(0), blocks(min(grid, total_)), step(0)
    {
        if (total / kTreeDrawnTiles < grid) return;
        length = total / blocks * 11 / 16;
        drawn = length * blocks;
        const int pieces = short_pieces * blocks;
        step = (total - drawn + pieces - 1) / pieces;
    }
    __device__ __forceinline__ int count() const { return step == 0 ? blocks : blocks + (total - drawn + step - 1) / step; }
    __device__ __forceinline__ int first(int c) const
    {
        // (equal shares: the first total % blocks ones are one tile longer)
        if (step == 0) return c < blocks ? total / blocks * c + min(c, total % blocks) : total;
        return c <= blocks ? length * c : min(total, drawn + (c - blocks) * step);
    }
};

// Tiles [t0, t1) of the n_tiles of one item; b < 0: no more.  `slot`: where its partial result goes: what starts
// inside an item goes to its piece's first slot, what ends inside one to its second.
struct TreeSegment {
    int b, len, nodes, hk, rb, t0, t1, n_tiles, slot;
    // Row 0 of the item's output and log-sum-exp: the caller's buffers, or the partial result's slot.  (Looked up by
    // the producer: at a segment's end the others would wait for the parameters.)
    void *out;
    float *lse;
    __device__ __forceinline__ bool whole() const { return t0 == 0 && t1 == n_tiles; }
    __device__ __forceinline__ int prefix() const { return len - nodes; }
};
static_assert(sizeof(TreeSegment) == kTreeEntryBytes, "queue entry");

// Draws this block's pieces and finds their segments (all 32 lanes of one warp together).  Out of line: the kernel's
// loops should stay in the instruction cache.
struct TreeFinder {
    TreePieces pieces;
    int n_pieces, piece, tile, end;
    unsigned drawn;                // lane 0: the next piece, asked for when this one began
    int b, len, nodes;             // a sequence with tiles ...
    int base, limit;               // ... the row's tiles [base, limit)
    __device__ __forceinline__ TreeFinder() : pieces(0, 1, 1) {}
    __device__ __noinline__ void start(const TreeParams &p, int total, int lane)
    {
        pieces = TreePieces(total, gridDim.x, p.short_pieces);
        n_pieces = pieces.count();
        b = -1;
        len = nodes = base = limit = 0;
        begin(p, (int)blockIdx.x < pieces.blocks ? blockIdx.x : n_pieces, lane);
    }
    __device__ __forceinline__ void begin(const TreeParams &p, int which, int lane)
    {
        piece = min(which, n_pieces);
        tile = end = 0;
        drawn = n_pieces;
        if (piece >= n_pieces) return;
        tile = pieces.first(piece);
        end = pieces.first(piece + 1);
        if (lane == 0 && pieces.step > 0) drawn = pieces.blocks + atomicAdd(p.ticket, 1u);
    }
    template <int D>
    __device__ __noinline__ TreeSegment next(const TreeParams &p, int lane)
    {
        TreeSegment s;
        s.b = -1;
        const int items = p.a.heads * p.row_blocks;
        do {
            if (tile >= end && piece < n_pieces) {
                const unsigned got = __shfl_sync(0xffffffffu, drawn, 0);
                begin(p, got < (unsigned)n_pieces ? (int)got : n_pieces, lane);
            }
            if (piece >= n_pieces) return s;
            while (tile >= limit) {    // (tile < W: some sequence has it)
                const int from = b + 1;
                if (from >= p.batch) return s;
                int n = 0, l = 0;
                if (from + lane < p.batch) l = checked_tree(p.tree, p.a.seq_lens, p.a.max_seq_len, nullptr, from + lane, false, n);
                const int mine = tree_weight(tree_tiles(l, n)) * items;
                int sum = mine;
#pragma unroll
                for (int o = 1; o < 32; o <<= 1) {
                    const int up = __shfl_up_sync(0xffffffffu, sum, o);
                    if (lane >= o) sum += up;
                }
                const unsigned reached = __ballot_sync(0xffffffffu, limit + sum > tile);
                const int at = reached ? __ffs(reached) - 1 : 31;
                len = __shfl_sync(0xffffffffu, l, at);
                nodes = __shfl_sync(0xffffffffu, n, at);
                base = limit + __shfl_sync(0xffffffffu, sum - mine, at);
                limit = limit + __shfl_sync(0xffffffffu, sum, at);
                b = from + at;
            }
            s.n_tiles = tree_tiles(len, nodes);
            if (b >= p.batch || s.n_tiles == 0) return s;     // (lengths that change under the kernel's hands)
            const int weight = tree_weight(s.n_tiles), inside = tile - base, item = inside / weight;
            const int from = inside - item * weight;
            int to = min(weight, from + (end - tile));
            s.hk = item / p.row_blocks;
            s.rb = item - s.hk * p.row_blocks;
            s.t0 = max(0, from - kTreeItemCost);
            // An item that is short next to the long pieces and starts in one stays whole, with the piece that has its start.
            if (pieces.step > 0 && 2 * weight <= pieces.length && tile - from < pieces.drawn) {
                to = weight;
                if (from > 0) s.t0 = weight;                  // another piece has it
            }
            s.t1 = to - kTreeItemCost;
            tile += to - from;
        } while (s.t1 <= s.t0);                               // only of the item's extra weight
        s.b = b;
        s.len = len;
        s.nodes = nodes;
        if (lane == 0) {
            int2 *of_item = p.item_pieces + (int64_t)b * items + s.hk * p.row_blocks + s.rb;
            if (s.t0 == 0) of_item->x = piece;
            if (s.t1 == s.n_tiles) of_item->y = piece;
        }
        s.slot = 2 * piece + (s.t0 == 0 ? 1 : 0);
        const int64_t row = (int64_t)b * p.tree.tokens * (p.a.heads * p.group) + s.hk * p.group, slot_row = (int64_t)s.slot * p.item_rows;
        s.out = s.whole() ? static_cast<void *>(p.a.out + row * D) : static_cast<void *>(p.a.part_o + slot_row * D);
        s.lse = !s.whole() ? p.a.part_lse + slot_row : p.a.lse ? p.a.lse + row : nullptr;
        return s;
    }
};

// The announced segments, for the warps that work on them: segment k of the block is entry k % 4.
struct TreeQueue {
    unsigned misc;
    unsigned char *misc_ptr;
    __device__ __forceinline__ TreeSegment &entry(int k) const { return reinterpret_cast<TreeSegment *>(misc_ptr + kTreeSegments)[k & 3]; }
    // Waits for segment k (all lanes); false if the wait ran out.
    __device__ __forceinline__ bool wait(int k) const
    {
        return __all_sync(0xffffffffu, tree_wait(misc + kTreeBarSegFull + (k & 3) * 8, (k >> 2) & 1));
    }
    __device__ __forceinline__ void done(int k, int lane) const
    {
        __syncwarp();
        if (lane == 0) mbarrier_arrive(misc + kTreeBarSegEmpty + (k & 3) * 8);
    }
};

// Adds up all sequences' tiles and leaves the sum in the misc region (all threads; the caller synchronises).
__device__ __forceinline__ void tree_count_tiles(const TreeParams &p, unsigned char *misc_ptr, int threads)
{
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    int mine = 0;                      // (all tiles are fewer than 2^31: checked by the host)
    for (int b = threadIdx.x; b < p.batch; b += threads) {
        int nodes;
        const int len = checked_tree(p.tree, p.a.seq_lens, p.a.max_seq_len, p.a.status, b, blockIdx.x == 0, nodes);
        mine += tree_weight(tree_tiles(len, nodes));
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) mine += __shfl_xor_sync(0xffffffffu, mine, o);
    int *scan = reinterpret_cast<int *>(misc_ptr + kTreeScan);
    if (lane == 0) scan[warp] = mine;
    __syncthreads();
    if (threadIdx.x == 0) {
        int total = 0;
        for (int w = 0; w < threads / 32; ++w) total += scan[w];
        *reinterpret_cast<int *>(misc_ptr + kTreeTotal) = total * p.a.heads * p.row_blocks;
    }
}

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

// 32 bytes to a 32-byte boundary.
__device__ __forceinline__ void store_32b(void *to, const unsigned (&v)[8])
{
    asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};"
                 :: "l"(to), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]) : "memory");
}

// Two 32-bit operations in one instruction.
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c)
{
    uint64_t x, y, z, d;
    asm("mov.b64 %0, {%1, %2};" : "=l"(x) : "f"(a.x), "f"(a.y));
    asm("mov.b64 %0, {%1, %2};" : "=l"(y) : "f"(b.x), "f"(b.y));
    asm("mov.b64 %0, {%1, %2};" : "=l"(z) : "f"(c.x), "f"(c.y));
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(x), "l"(y), "l"(z));
    float2 r;
    asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(d));
    return r;
}
__device__ __forceinline__ float2 add2(float2 a, float2 b)
{
    uint64_t x, y, d;
    asm("mov.b64 %0, {%1, %2};" : "=l"(x) : "f"(a.x), "f"(a.y));
    asm("mov.b64 %0, {%1, %2};" : "=l"(y) : "f"(b.x), "f"(b.y));
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(x), "l"(y));
    float2 r;
    asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(d));
    return r;
}

__device__ __forceinline__ float max3(float a, float b, float c)
{
    float d;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
    return d;
}
// The largest of 32 values and `top`, as two chains (NaN does not count).
__device__ __forceinline__ float max32(const float (&x)[32], float top)
{
    float even = max3(top, x[0], x[1]), odd = fmaxf(x[2], x[3]);
#pragma unroll
    for (int c = 4; c < 32; c += 4) {
        even = max3(even, x[c], x[c + 1]);
        odd = max3(odd, x[c + 2], x[c + 3]);
    }
    return fmaxf(even, odd);
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


// The copies of one block: K and V tiles into their rings, the query rows, and the clean-up of value rows
// that must not meet a weight of 0.  `ring` and `misc` are shared-memory addresses, smem the ring's pointer.
template <int D, bool kPaged, typename Ring>
struct TreeCopies {
    const TreeParams &p;
    unsigned char *smem;
    unsigned ring, misc;
    int lane;

    __device__ __forceinline__ int run_tokens() const { return kPaged ? min(p.a.block_tokens, kTreeTile) : kTreeTile; }
    // lane i: the physical block of the i-th run of tile j
    __device__ __forceinline__ int fetch_ids(const TreeSegment &s, int j) const
    {
        if (!kPaged) return 0;
        const int T = run_tokens(), start = j * kTreeTile;
        if (j >= s.t1 || lane >= (min(s.len - start, kTreeTile) + T - 1) / T) return -1;
        const int idx = (start + lane * T) / p.a.block_tokens;
        if (!bounds_ok(idx < p.a.max_blocks_per_seq, p.a.status)) return -1;
        return p.a.block_table[(int64_t)s.b * p.a.max_blocks_per_seq + idx];
    }
    // One tile of one cache (all lanes); false if a wait ran out.
    template <bool kIsV>
    __device__ __forceinline__ bool copy_tile(const TreeSegment &s, int j, int phys, const CUtensorMap *map, int &count) const
    {
        constexpr int slots = kIsV ? Ring::kVSlots : Ring::kKSlots, ring_offset = kIsV ? Ring::kVOffset : 0;
        constexpr int bar_full = kIsV ? kTreeBarVFull : kTreeBarKFull, bar_empty = kIsV ? kTreeBarVEmpty : kTreeBarKEmpty;
        const AttnParams &a = p.a;
        const int T = run_tokens(), start = j * kTreeTile;
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
        for (int item = 0; item < Ring::kItems; ++item, ++count) {
            const int slot = count % slots;
            if (count >= slots &&
                !__all_sync(0xffffffffu, tree_wait(misc + bar_empty + slot * 8, (count / slots - 1) & 1)))
                return false;
            const int slot_offset = ring_offset + slot * Ring::kItemBytes + (kPaged ? lane * T * 128 : 0);
            const unsigned bar = misc + bar_full + slot * 8;
            if (kPaged && lane < nb && !good) {                   // a block that cannot be read counts as zeros
                const uint4 zero = make_uint4(0u, 0u, 0u, 0u);
#pragma unroll 1
                for (int i = 0; i < T * 8; ++i) {
#pragma unroll
                    for (int panel = 0; panel < Ring::kItemPanels; ++panel)
                        *reinterpret_cast<uint4 *>(smem + slot_offset + panel * kTreePanelBytes + i * 16) = zero;
                }
                fence_async_proxy();
            }
            __syncwarp();                                // (where no copy is left to wait for, the arrival alone completes the item)
            if (lane == 0) mbarrier_expect_bytes(bar, fetched * (unsigned)(T * 128 * Ring::kItemPanels));
            __syncwarp();
            if (good) {
#pragma unroll
                for (int panel = 0; panel < Ring::kItemPanels; ++panel)
                    tma_load_2d(ring + slot_offset + panel * kTreePanelBytes, map, (item * Ring::kItemPanels + panel) * 64, row0, bar);
            }
        }
        return true;
    }
    // copies in flight must land (or be given up, bounded) before shared memory is handed on
    template <bool kIsV>
    __device__ __forceinline__ void drain(int count) const
    {
        constexpr int slots = kIsV ? Ring::kVSlots : Ring::kKSlots, bar_full = kIsV ? kTreeBarVFull : kTreeBarKFull;
        for (int i = max(count - slots, 0); i < count; ++i)
            (void)tree_wait(misc + bar_full + (i % slots) * 8, (i / slots) & 1);
    }
    // The K producer's whole job: draws the pieces, announces their segments, copies the K tiles, and behind the
    // first tile of every segment its query rows, kBlocks row blocks (64 dims of one per kQPanel bytes) at q_smem.
    template <int kBlocks, int kQPanel>
    __device__ __forceinline__ void produce_k(const TreeQueue &queue, const CUtensorMap *map_q, const CUtensorMap *map_k, unsigned q_smem) const
    {
        TreeFinder finder;
        finder.start(p, *reinterpret_cast<const int *>(queue.misc_ptr + kTreeTotal), lane);
        int count = 0, k = 0;
        bool fine = true;
        // Segments are found two ahead, while the copies of the one before wait for their slots: lengths, block ids
        // and the ticket's answer come from a busy memory system, some 2000 cycles each.
        auto announce = [&](const TreeSegment &s, int n) -> bool {
            if (n >= 4 && !__all_sync(0xffffffffu, tree_wait(misc + kTreeBarSegEmpty + (n & 3) * 8, ((n >> 2) - 1) & 1))) return false;
            if (lane == 0) {
                queue.entry(n) = s;
                mbarrier_arrive(misc + kTreeBarSegFull + (n & 3) * 8);
            }
            return true;
        };
        TreeSegment seg = finder.template next<D>(p, lane);
        (void)announce(seg, 0);
        int ids = seg.b >= 0 ? fetch_ids(seg, seg.t0) : -1;
        TreeSegment after = seg;
        if (seg.b >= 0) {
            after = finder.template next<D>(p, lane);
            (void)announce(after, 1);
        }
        for (; fine && seg.b >= 0; ++k) {
            TreeSegment later = after;                // segment k + 2
            int ids_after = -1;
            for (int j = seg.t0; j < seg.t1 && fine; ++j) {
                const int now = ids;
                ids = fetch_ids(seg, j + 1);
                fine = copy_tile<false>(seg, j, now, map_k, count);
                if (j > seg.t0 || !fine) continue;
                // the query rows wait for the last segment's logits
                if (k >= 1) fine = __all_sync(0xffffffffu, tree_wait(misc + kTreeBarQEmpty, (k - 1) & 1));
                if (fine && lane == 0) {
                    const int panel_bytes = p.nodes_per_block * p.group * 128;
                    int blocks = 0;
#pragma unroll
                    for (int s = 0; s < kBlocks; ++s) blocks += (seg.rb * kBlocks + s) * p.nodes_per_block < p.tree.tokens;
                    mbarrier_expect_bytes(misc + kTreeBarQFull, (unsigned)(blocks * panel_bytes * Ring::kPanels));
#pragma unroll
                    for (int s = 0; s < kBlocks; ++s) {
                        const int node0 = (seg.rb * kBlocks + s) * p.nodes_per_block;
                        if (node0 >= p.tree.tokens) continue;
#pragma unroll
                        for (int panel = 0; panel < Ring::kPanels; ++panel)
                            tma_load_4d(q_smem + (s * Ring::kPanels + panel) * kQPanel, map_q, panel * 64, seg.hk * p.group, node0,
                                        seg.b, misc + kTreeBarQFull);
                    }
                }
                __syncwarp();
                if (after.b >= 0) {
                    ids_after = fetch_ids(after, after.t0);
                    later = finder.template next<D>(p, lane);
                    fine = fine && announce(later, k + 2);
                }
            }
            if (!fine) break;
            seg = after;
            after = later;
            ids = ids_after;
        }
        if (!fine) {
            if (lane == 0 && p.a.status) atomicOr(p.a.status, kFlagCopyTimeout);
            drain<false>(count);
            (void)tree_wait(misc + kTreeBarQFull, k & 1);     // (the query rows of this segment, if they were asked for)
        }
    }
    __device__ __forceinline__ void produce_v(const TreeQueue &queue, const CUtensorMap *map_v) const
    {
        int count = 0, k = 0;
        bool fine = queue.wait(0);
        auto take = [&](int n) -> TreeSegment {
            const TreeSegment s = queue.entry(n);
            queue.done(n, lane);
            return s;
        };
        TreeSegment seg;
        seg.b = -1;
        if (fine) seg = take(0);
        int ids = seg.b >= 0 ? fetch_ids(seg, seg.t0) : -1;
        for (; fine && seg.b >= 0; ++k) {
            TreeSegment after;
            bool have = false;                        // the next segment is announced by now, and its first ids are asked for
            int ids_after = -1;
            for (int j = seg.t0; j < seg.t1 && fine; ++j) {
                const int now = ids;
                ids = fetch_ids(seg, j + 1);
                fine = copy_tile<true>(seg, j, now, map_v, count);
                if (!have && fine) have = __all_sync(0xffffffffu, mbarrier_test(misc + kTreeBarSegFull + ((k + 1) & 3) * 8, ((k + 1) >> 2) & 1));
                else continue;
                if (have) {
                    after = take(k + 1);
                    if (after.b >= 0) ids_after = fetch_ids(after, after.t0);
                }
            }
            if (!have && fine) {
                fine = queue.wait(k + 1);
                if (!fine) break;
                after = take(k + 1);
                if (after.b >= 0) ids_after = fetch_ids(after, after.t0);
            }
            seg = after;
            ids = ids_after;
        }
        if (!fine) {
            if (lane == 0 && p.a.status) atomicOr(p.a.status, kFlagCopyTimeout);
            drain<true>(count);
        }
    }
    // Rows row0 .. row0 + kRows - 1 of the V tile number g of this block (one warp).  Value rows behind the sequence get
    // weight 0 but may hold anything, and 0 x NaN is NaN: they are cleared.  A node's row that is not finite is
    // cleared too and noted in `poison`; the rows that see it get it added at the end.
    template <int kRows>
    __device__ __forceinline__ void clean_values(const TreeSegment &s, int j, int g, int row0, unsigned *poison, bool &fine) const
    {
        const int start = j * kTreeTile + row0;
        if (start + kRows - 1 < s.prefix()) return;                          // uniform
        unsigned char *rows[Ring::kItems];
#pragma unroll
        for (int item = 0; item < Ring::kItems; ++item) {
            const int n = g * Ring::kItems + item, slot = n % Ring::kVSlots;
            if (fine) fine = tree_wait(misc + kTreeBarVFull + slot * 8, (n / Ring::kVSlots) & 1);
            rows[item] = smem + Ring::kVOffset + slot * Ring::kItemBytes + row0 * 128;
        }
        __syncwarp();
        unsigned bad_rows = 0;
#pragma unroll 1
        for (int r0 = 0; r0 < kRows; r0 += 4) {                       // four rows at a time, 8 lanes a row
            const int pos = start + r0 + (lane >> 3);
            bool bad = false;
#pragma unroll
            for (int i = 0; i < Ring::kPanels; ++i)
                bad = bad || !finite8(*reinterpret_cast<const uint4 *>(rows[i / Ring::kItemPanels] + i % Ring::kItemPanels * kTreePanelBytes +
                                                                       r0 * 128 + lane * 16));
            const unsigned found = __ballot_sync(0xffffffffu, bad && pos >= s.prefix() && pos < s.len);
            const bool mine = (found >> (lane & 24) & 0xffu) != 0;
            if (mine || pos >= s.len) {
#pragma unroll
                for (int i = 0; i < Ring::kPanels; ++i)
                    *reinterpret_cast<uint4 *>(rows[i / Ring::kItemPanels] + i % Ring::kItemPanels * kTreePanelBytes + r0 * 128 +
                                               lane * 16) = make_uint4(0u, 0u, 0u, 0u);
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) bad_rows |= (unsigned)((found >> (8 * i) & 0xffu) != 0) << (r0 + i);
        }
        fence_async_proxy();
        if (lane == 0) {
            for (; bad_rows != 0; bad_rows &= bad_rows - 1) {
                const int node = start + __ffs(bad_rows) - 1 - s.prefix();
                atomicOr(poison + (node >> 5), 1u << (node & 31));
            }
        }
        __syncwarp();
    }
};

// Value rows that were taken out of their tiles (rare), given back to the rows that see them.
// The weight of cache row kv_row for query row out_row, against that row's log-sum-exp.
__device__ __forceinline__ float tree_stray_weight(const AttnParams &a, int64_t out_row, int64_t kv_row, int D, float lse2)
{
    float dot = 0.f;
    #pragma unroll 1
    for (int c = 0; c < D; ++c) dot = fmaf(__half2float(a.q[out_row * D + c]), __half2float(a.k[kv_row * D + c]), dot);
    return fast_exp2(dot * a.scale_log2e - lse2);
}
// Adds what `row` sees of them to its dims d0 .. d0 + 31 in o.
static __device__ __noinline__ void tree_add_poisoned(const AttnParams &a, const TreeSegment &s, const TreeRow &row, const unsigned *poison,
                                               int64_t out_row, int D, int d0, float lse2, float *o)
{
    for (int n = 0; n < s.nodes; ++n) {
        if (!(poison[n >> 5] >> (n & 31) & 1u) || !row.sees(n)) continue;
        const int64_t kv_row = tree_cache_row(a, s.b, s.hk, s.prefix() + n);
        const float weight = tree_stray_weight(a, out_row, kv_row, D, lse2);
#pragma unroll 1
        for (int c = 0; c < 32; ++c) o[c] += weight * __half2float(a.v[kv_row * D + d0 + c]);
    }
}
// Dim d of what row r of a segment's only row block sees of them (the kernel with the tokens as the long side).
static __device__ __noinline__ float tree_poisoned_value(const TreeParams &p, const TreeSegment &s, const unsigned *poison, int r, int D, int d,
                                                  float lse2)
{
    const AttnParams &a = p.a;
    const int node = r / p.group;
    const TreeRow row = tree_row(p.tree, s.b, node, s.nodes);
    const int64_t out_row = ((int64_t)s.b * p.tree.tokens + node) * ((int64_t)a.heads * p.group) + (int64_t)s.hk * p.group + (r - node * p.group);
    float value = 0.f;
    for (int n = 0; n < s.nodes; ++n) {
        if (!(poison[n >> 5] >> (n & 31) & 1u) || !row.sees(n)) continue;
        const int64_t kv_row = tree_cache_row(a, s.b, s.hk, s.prefix() + n);
        value += tree_stray_weight(a, out_row, kv_row, D, lse2) * __half2float(a.v[kv_row * D + d]);
    }
    return value;
}

// The barriers that the kernels have in common, and the poison words (one thread); softmax_warps: how many work on
// one unit of logits.
__device__ __forceinline__ void tree_init_barriers(unsigned misc, unsigned char *misc_ptr, int softmax_warps, int all_softmax_warps)
{
#pragma unroll
    for (int s = 0; s < 6; ++s) {
        mbarrier_init(misc + kTreeBarKFull + s * 8, 1);
        mbarrier_init(misc + kTreeBarKEmpty + s * 8, 1);
        mbarrier_init(misc + kTreeBarVFull + s * 8, 1);
        mbarrier_init(misc + kTreeBarVEmpty + s * 8, 1);
    }
#pragma unroll
    for (int s = 0; s < 4; ++s) {
        mbarrier_init(misc + kTreeBarSFull + s * 8, 1);
        mbarrier_init(misc + kTreeBarPFull + s * 8, softmax_warps);
        mbarrier_init(misc + kTreeBarPvDone + s * 8, 1);
        if (s < 2) mbarrier_init(misc + kTreeBarSFree + s * 8, softmax_warps);
    }
#pragma unroll
    for (int s = 0; s < 4; ++s) {
        mbarrier_init(misc + kTreeBarSegFull + s * 8, 1);
        mbarrier_init(misc + kTreeBarSegEmpty + s * 8, all_softmax_warps + 3);     // V producer and the two MMA issuers too
    }
    mbarrier_init(misc + kTreeBarQFull, 1);
    mbarrier_init(misc + kTreeBarQEmpty, 1);
    mbarrier_init_fence();
    for (int i = 0; i < 32; ++i) reinterpret_cast<unsigned *>(misc_ptr + kTreePoison)[i] = 0u;
}

// Joins the partial results of the items that more than one piece has a part of, and zeroes the rows of
// sequences without work; a block takes kTreeMergeRows rows of an item, a warp one after the other of them.  The work is a chain of short loads (the item's pieces, their
// log-sum-exps, the partials), so each link is one round of loads: a lane per piece, then eight partials at a time.
constexpr int kTreeMergeThreads = 256;
constexpr int kTreeMergeRows = 32;

template <int D>
__global__ void __launch_bounds__(kTreeMergeThreads)
tree_merge_kernel(const TreeParams p, int row_parts)
{
    const AttnParams &a = p.a;
    const int lane = threadIdx.x & 31;
    const int part = blockIdx.x % row_parts, item = blockIdx.x / row_parts;           // (sequence, KV head, row block)
    const int items = a.heads * p.row_blocks;
    const int b = item / items, in_seq = item - b * items;
    const int hk = in_seq / p.row_blocks, rb = in_seq - hk * p.row_blocks;
    allow_next_kernel();
    wait_for_previous_kernels();
    int nodes;
    const int2 pieces = p.item_pieces[item];
    const int len = checked_tree(p.tree, a.seq_lens, a.max_seq_len, nullptr, b, false, nodes);
    const int c0 = pieces.x, n = tree_tiles(len, nodes) > 0 ? pieces.y - c0 + 1 : 0;
    if (n == 1) return;                                               // one piece had it all: the result is written
#pragma unroll 1
    for (int in_part = threadIdx.x >> 5; in_part < kTreeMergeRows; in_part += kTreeMergeThreads / 32) {
        const int r = part * kTreeMergeRows + in_part;
        const int node = rb * (p.item_rows / p.group) + r / p.group, head = r % p.group;
        if (r >= p.item_rows || node >= p.tree.tokens) break;
        const int64_t out_row = ((int64_t)b * p.tree.tokens + node) * ((int64_t)a.heads * p.group) + (int64_t)hk * p.group + head;
        // (the item's start went to its piece's second slot, all else to the first one)
        auto slot_row = [&](int i) -> int64_t { return (int64_t)(2 * (c0 + i) + (i == 0 ? 1 : 0)) * p.item_rows + r; };
        float top = kMinusHuge, total = 0.f;
        bool any_nan = false;
        for (int i = lane; i < n; i += 32) {
            const float lse = a.part_lse[slot_row(i)];
            top = fmaxf(top, lse);
            any_nan = any_nan || lse != lse;
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
        const bool empty = !(top > kMinusHuge) && !__any_sync(0xffffffffu, any_nan);
        // A lane's dims: kVecs runs of kWidth.
        constexpr int kPer = D / 32, kVecs = kPer >= 4 ? kPer / 4 : 1, kWidth = kPer / kVecs, kDeep = 8 / kVecs;
        float acc[kPer];
#pragma unroll
        for (int i = 0; i < kPer; ++i) acc[i] = 0.f;
        for (int i0 = 0; i0 < n && !empty; i0 += 32) {
            const float mine = i0 + lane < n ? fast_exp2(a.part_lse[slot_row(i0 + lane)] - top) : 0.f;
            const int here = min(32, n - i0);
            for (int i = 0; i < here; i += kDeep) {
                float x[kDeep][kPer];
#pragma unroll
                for (int u = 0; u < kDeep; ++u) {
                    if (i + u < here) {
                        const float *from = a.part_o + slot_row(i0 + i + u) * D + lane * kWidth;
#pragma unroll
                        for (int v = 0; v < kVecs; ++v) {
                            if constexpr (kWidth == 4) *reinterpret_cast<float4 *>(&x[u][4 * v]) = *reinterpret_cast<const float4 *>(from + v * 128);
                            else *reinterpret_cast<float2 *>(&x[u][0]) = *reinterpret_cast<const float2 *>(from);
                        }
                    }
                }
#pragma unroll
                for (int u = 0; u < kDeep; ++u) {
                    const float w = __shfl_sync(0xffffffffu, mine, (i + u) & 31);
                    if (i + u < here) {
                        total += w;
#pragma unroll
                        for (int d = 0; d < kPer; ++d) acc[d] = fmaf(w, x[u][d], acc[d]);
                    }
                }
            }
        }
        const float inverse = empty ? 0.f : 1.f / total;
        unsigned *to = reinterpret_cast<unsigned *>(a.out + out_row * D);
#pragma unroll
        for (int i = 0; i < kPer; i += 2) {
            const int d = lane * kWidth + i / 4 * 128 + i % 4;            // (kWidth 2: i is 0)
            to[d / 2] = empty ? 0u : pack_half2(acc[i] * inverse, acc[i + 1] * inverse);
        }
        if (a.lse && lane == 0) a.lse[out_row] = empty ? -INFINITY : (top + log2f(total)) * kLn2;
    }
}

}  // namespace instinfer
