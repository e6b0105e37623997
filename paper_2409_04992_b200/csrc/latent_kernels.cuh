// Decode attention over a latent cache on the fifth-generation tensor cores, for sm_100a.
//
// A cache row is one token's latent vector c (L dims, shared by all heads) and its turned key part (64 dims); a query
// row is a head's absorbed query of the same width.  All heads attend to the same rows, and the values are the rows'
// first L dims:
//   out[r] = softmax_i(scale q[r] . [c_i, k_i]) . c_i
// so R = new tokens x heads query rows share every byte of the cache: 2 R (2 L + 64) operations for 2 (L + 64) bytes.
//
// The TOKENS are the long side of the MMAs, N = 16 or 32 rows the short one, and both products read the one tile of
// 64 tokens that lies in shared memory, row-major for the first and column-major for the second:
//   S^T[64 tokens x N]     = tile[64 x (L + 64)] Q^T[(L + 64) x N]
//   O^T[128 dims x N] (L / 128 accumulators) += tile^T[128 x 64] P^T[64 x N]
// More than 32 rows take pairs of SMs (latent_pair_kernels.cuh).  Those cut more than 128 rows into row blocks; the pairs of a
// "plane" take one row block each, their tiles cut alike, so that the pairs of all planes that work on the same tokens run
// at about the same time and all but the first find them in L2.
//
// Work split: a plane's tiles, item after item (an item is a row block of a sequence), lie in one row that is cut into
// equal shares, one per block.  Only the items that a share starts or ends inside leave partial results, two per block at
// most.  (Shorter pieces drawn from a counter, which the kernels for draft trees take, lose here: a partial result is four
// times as large and each of its segments costs some three tiles; 128 sequences of 16k, 16 heads: 408 us with equal
// shares, 465 with four drawn pieces a block.)  An item counts some tiles more than it has, for its segment's set-up.
//
// Measured: 16 rows, 64 sequences of 4k to 16k tokens in 64-token pages 140 us (5.4 TB/s), 128 of 16k 412 us (5.9 TB/s); 32 rows,
// 32 sequences of 8k 71 us; one sequence of 1000 tokens 14 us, a chain of set-up, one tile and the merge.
//
// A block has four softmax warps and three single-purpose warps that hand tiles over through mbarriers, as in the kernels
// for draft trees:
//   producer                 finds the share's segments (its parts of items), announces them through a queue in shared
//                            memory, copies tiles (64-dim panels by tensor-map copies, 128-byte swizzle) and query rows;
//   logit and output issuer  one elected thread each issues the MMAs.  An item (128 dims of the tile) goes back to the producer as
//                            soon as its accumulator's MMAs are complete, the turned part after the logits'.
// A thread of the softmax warps has two tokens and a quarter of the rows (the 16-lane shape of the tensor-memory
// load: 64 tokens fill 16 lanes of every warp's 32).  References are logits before the scale and follow the maximum
// lazily, weights enter the second product as 16-bit high and low parts, and sums are 32-bit: as in tree_umma_tokens.cuh,
// which has the reasons.
#pragma once

#include <type_traits>

#include "tree_umma_tokens.cuh"

namespace instinfer {

constexpr int kLatentTile = 64;                          // tokens per tile
constexpr int kLatentRope = 64;                          // turned dims
constexpr int kLatentPanel = kLatentTile * 128;          // 64 dims of a tile
constexpr int kLatentItem = 2 * kLatentPanel;            // 128 dims

struct LatentParams {
    TreeShape tree;              // mask == nullptr: a chain, node t sees nodes 0 .. t
    const int32_t *seq_lens;
    const int32_t *block_table;  // nullptr: contiguous
    int32_t *status;
    const void *cache;
    void *out;                   // [batch, rows, L]
    float *lse;                  // nullable [batch, rows]
    float *part_o;               // [slots, block_rows, L]
    float *part_lse;             // [slots, block_rows]
    int2 *item_shares;           // [batch * row_blocks] the shares with an item's first and last tile, for the merge
    int64_t num_phys_blocks;
    int64_t cache_rows;
    int32_t batch;
    int32_t q_heads;
    int32_t rows;                // query rows of a sequence: new tokens x heads
    int32_t block_rows;          // of a row block (the last one may have fewer)
    int32_t row_blocks;
    int32_t planes;
    int32_t teams;               // blocks (or pairs of blocks) of a plane
    int32_t tile_shift;          // tokens of a tile: 2^tile_shift
    int32_t item_cost;           // what a segment's set-up and end count in tiles
    int32_t max_seq_len;
    int32_t s_max;
    int32_t block_tokens;
    int32_t run_tokens;          // a tile is 64 / run_tokens copies per panel: consecutive rows of one block
    int32_t max_blocks_per_seq;
    float scale, scale_log2e;
};

// Offsets inside the misc region.
constexpr int kLatBarFull = 0;         // [12] an item landed
constexpr int kLatBarEmpty = 96;       // [12]
constexpr int kLatBarRopeFull = 192;   // [4]
constexpr int kLatBarRopeEmpty = 224;  // [4]
constexpr int kLatBarSFull = 256;      // [2] logits of a tile are in tensor memory
constexpr int kLatBarSFree = 272;      // [2]
constexpr int kLatBarPFull = 288;      // its weights are in shared memory
constexpr int kLatBarPvDone = 296;     // its output MMAs are complete
constexpr int kLatBarQFull = 304;
constexpr int kLatBarQEmpty = 312;
constexpr int kLatBarSegFull = 320;    // [4]
constexpr int kLatBarSegEmpty = 352;   // [4]
constexpr int kLatTmemPtr = 384;
constexpr int kLatTotal = 388;         // the plane's tiles; a window's first sequence and its start
constexpr int kLatScan = 400;          // [16] ints, before the first segment
constexpr int kLatSegments = 464;      // [4] LatentSegment
constexpr int kLatSegmentBytes = 56;
constexpr int kLatMiscBytes = 704;
static_assert(kLatSegments + 4 * kLatSegmentBytes <= kLatMiscBytes && kLatScan + 64 <= kLatSegments, "misc region too small");

template <int L, int N>
struct LatentGeometry {
    static_assert(L == 512 && (N == 16 || N == 32), "instances");
    static constexpr int kPanels = L / 64;                               // latent panels of a tile; the turned part is one more
    static constexpr int kItems = L / 128;
    static constexpr int kQPanel = N * 128;
    static constexpr int kQBytes = (kPanels + 1) * kQPanel;
    static constexpr int kPPart = N * kLatentTile * 2;                   // weights of a tile: high parts, then low parts
    static constexpr int kThreads = (4 + 3) * 32;
    static constexpr int kExtraBytes = kLatMiscBytes + N * 20;           // a row's numbers by warp, and its reference
    static constexpr int kRoom = 226 * 1024 - kQBytes - 2 * kPPart - kExtraBytes;
    static constexpr int kTiles = kRoom / (kItems * kLatentItem + kLatentPanel);     // whole tiles that fit
    static constexpr int kRopeSlots = kTiles < 4 ? kTiles : 4;
    static constexpr int kSlots = (kRoom - kRopeSlots * kLatentPanel) / kLatentItem;
    static constexpr int kRopeOffset = kSlots * kLatentItem;
    static constexpr int kQOffset = kRopeOffset + kRopeSlots * kLatentPanel;
    static constexpr int kPOffset = kQOffset + kQBytes;
    static constexpr int kMiscOffset = kPOffset + 2 * kPPart;
    static constexpr int kSmemBytes = kMiscOffset + kExtraBytes + 1024;  // room to align to 1024 bytes
    // The low parts are further columns of the same MMAs, whose time is that of reading the tile.
    static constexpr int kAccCols = 2 * N;
    static constexpr int kOColumn = 2 * N;                               // two logit buffers, then the accumulators
    static constexpr int kUsedCols = kOColumn + kItems * kAccCols;
    static constexpr int kTmemCols = kUsedCols > 256 ? 512 : kUsedCols > 128 ? 256 : 128;
    static_assert(kSlots >= 2 * kItems && kSlots <= 12 && kRopeSlots >= 1 && kRopeSlots <= 4 && kUsedCols <= 512, "rings, tensor memory");
    static_assert(kSmemBytes <= 227 * 1024, "one block per SM must fit");
};

// Tiles [t0, t1) of the n_tiles of one item; b < 0: no more.
struct LatentSegment {
    int b, len, nodes, row0, t0, t1, n_tiles, slot;      // row0: the item's first query row
    void *out;                                           // row 0 of its output and log-sum-exp: the caller's, or the slot's
    float *lse;
    int rows, pad;                                       // its query rows
    __device__ __forceinline__ bool whole() const { return t0 == 0 && t1 == n_tiles; }
    __device__ __forceinline__ int prefix() const { return len - nodes; }
};
static_assert(sizeof(LatentSegment) == kLatSegmentBytes, "queue entry");

__device__ __forceinline__ int latent_tiles(const LatentParams &p, int len, int nodes)
{
    return nodes > 0 ? (int)(((unsigned)len + (1u << p.tile_shift) - 1) >> p.tile_shift) : 0;
}
__device__ __forceinline__ int latent_weight(const LatentParams &p, int tiles) { return tiles > 0 ? tiles + p.item_cost : 0; }
// Row blocks of a sequence that a plane has: plane, plane + planes, ...
__device__ __forceinline__ int latent_plane_items(const LatentParams &p, int plane) { return (p.row_blocks - plane + p.planes - 1) / p.planes; }

// Finds the segments of this block's share (all 32 lanes of one warp together).
struct LatentFinder {
    int plane, items, team;        // the block's plane, row blocks of a sequence there, its number in it
    int tile, end;                 // what is left of the share
    // 32 sequences from w0 on, one a lane: length, new tokens, and where its items end in the plane's row; start: the first one's start
    int w0, start, len, nodes, stop;
    __device__ __forceinline__ void load(const LatentParams &p, int lane)
    {
        len = nodes = 0;
        if (w0 + lane < p.batch) len = checked_tree(p.tree, p.seq_lens, p.max_seq_len, nullptr, w0 + lane, false, nodes);
        stop = latent_weight(p, latent_tiles(p, len, nodes)) * items;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int up = __shfl_up_sync(0xffffffffu, stop, o);
            if (lane >= o) stop += up;
        }
        stop += start;
    }
    // The share of a plane of `total` tiles; the window lies at or before its first tile.
    __device__ __forceinline__ void begin(const LatentParams &p, int total)
    {
        const int blocks = min(p.teams, total);
        tile = end = total;
        if (team >= blocks) return;
        const int length = total / blocks, longer = total - length * blocks;       // (the first `longer` shares are one tile longer)
        tile = length * team + min(team, longer);
        end = tile + length + (team < longer ? 1 : 0);
    }
    template <typename E, int L>
    __device__ __noinline__ LatentSegment next(const LatentParams &p, int lane)
    {
        LatentSegment s;
        s.b = -1;
        for (;;) {
            if (tile >= end) return s;
            unsigned reached = __ballot_sync(0xffffffffu, stop > tile);
            while (reached == 0) {
                w0 += 32;
                if (w0 >= p.batch) return s;          // (lengths that change under the kernel's hands)
                start = __shfl_sync(0xffffffffu, stop, 31);
                load(p, lane);
                reached = __ballot_sync(0xffffffffu, stop > tile);
            }
            const int at = __ffs(reached) - 1;
            const int before = __shfl_sync(0xffffffffu, stop, max(at - 1, 0));
            s.len = __shfl_sync(0xffffffffu, len, at);
            s.nodes = __shfl_sync(0xffffffffu, nodes, at);
            s.n_tiles = latent_tiles(p, s.len, s.nodes);
            const int weight = latent_weight(p, s.n_tiles), inside = tile - (at == 0 ? start : before), item = items == 1 ? 0 : inside / weight;
            const int from = inside - item * weight, to = min(weight, from + (end - tile));
            const int rb = plane + item * p.planes;
            s.t0 = max(0, from - p.item_cost);
            s.t1 = to - p.item_cost;
            tile += to - from;
            if (s.t1 <= s.t0) continue;               // only of the item's extra weight
            s.b = w0 + at;
            s.row0 = rb * p.block_rows;
            s.rows = min(p.block_rows, p.rows - s.row0);
            s.pad = 0;
            if (lane == 0) {
                int2 *of_item = p.item_shares + (int64_t)s.b * p.row_blocks + rb;
                if (s.t0 == 0) of_item->x = team;
                if (s.t1 == s.n_tiles) of_item->y = team;
            }
            // (what starts inside an item goes to its block's first slot, what ends inside one to its second)
            s.slot = 2 * (plane + team * p.planes) + (s.t0 == 0 ? 1 : 0);
            const int64_t row = (int64_t)s.b * p.rows + s.row0, slot_row = (int64_t)s.slot * p.block_rows;
            s.out = s.whole() ? static_cast<void *>(static_cast<E *>(p.out) + row * L) : static_cast<void *>(p.part_o + slot_row * L);
            s.lse = !s.whole() ? p.part_lse + slot_row : p.lse ? p.lse + row : nullptr;
            return s;
        }
    }
};

// More than 32 sequences: all threads add up the plane's tiles (and report lengths out of range), and leave the total and
// where the window of 32 sequences around this block's first tile starts in the misc region.
__device__ __forceinline__ void latent_scan(const LatentParams &p, unsigned char *misc_ptr, int threads, int plane, int items, int team)
{
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int per = (p.batch + threads - 1) / threads, b0 = threadIdx.x * per;
    int mine = 0;                      // (all tiles are fewer than 2^31: checked by the host)
    for (int b = b0; b < min(b0 + per, p.batch); ++b) {
        int nodes;
        const int len = checked_tree(p.tree, p.seq_lens, p.max_seq_len, p.status, b, blockIdx.x == 0, nodes);
        mine += latent_weight(p, latent_tiles(p, len, nodes)) * items;
    }
    int sum = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int up = __shfl_up_sync(0xffffffffu, sum, o);
        if (lane >= o) sum += up;
    }
    int *scan = reinterpret_cast<int *>(misc_ptr + kLatScan);
    if (lane == 31) scan[warp] = sum;
    __syncthreads();
    int total = 0, before = 0;
    for (int w = 0; w < threads / 32; ++w) {
        if (w == warp) before = total;
        total += scan[w];
    }
    before += sum - mine;
    LatentFinder share;
    share.team = team;
    share.begin(p, total);
    int *found = reinterpret_cast<int *>(misc_ptr + kLatTotal);
    if (threadIdx.x == 0) found[0] = total;
    if (share.tile < share.end && before <= share.tile && share.tile < before + mine) {
        found[1] = b0;
        found[2] = before;
    }
}

// Lane i (row >= 0): brings the T cache rows from `row` on into L2.  (A hint: nothing waits for it.)
__device__ __forceinline__ void latent_prefetch(const LatentParams &p, int row, int T, int row_bytes)
{
    if (row < 0) return;
    const int64_t rows = min((int64_t)T, p.cache_rows - row);
    if (rows > 0)
        asm volatile("cp.async.bulk.prefetch.L2.global [%0], %1;"
                     :: "l"(static_cast<const char *>(p.cache) + (int64_t)row * row_bytes), "r"((unsigned)rows * (unsigned)row_bytes) : "memory");
}
__device__ __forceinline__ void tma_load_3d(unsigned dst, const CUtensorMap *map, int x, int y, int z, unsigned bar)
{
    asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes "
                 "[%0], [%1, {%2, %3, %4}], [%5];"
                 :: "r"(dst), "l"(reinterpret_cast<uint64_t>(map)), "r"(x), "r"(y), "r"(z), "r"(bar) : "memory");
}

// ---- the 16-lane shape of tensor memory: lane t of the warp gets columns 8 j + 2 (t % 4) + {0, 1} of rows t / 4 (v[4 j],
// v[4 j + 1]) and t / 4 + 8 (v[4 j + 2], v[4 j + 3]); valid after tc_loaded ----
template <int kRegs>
__device__ __forceinline__ void tc_issue_load_16lanes(float (&v)[kRegs], unsigned taddr)
{
    static_assert(kRegs == 8 || kRegs == 16, "16 or 32 columns");
    if constexpr (kRegs == 8)
        asm volatile("tcgen05.ld.sync.aligned.16x256b.x2.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                     : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]), "=f"(v[4]), "=f"(v[5]), "=f"(v[6]), "=f"(v[7])
                     : "r"(taddr) : "memory");
    else
        asm volatile("tcgen05.ld.sync.aligned.16x256b.x4.b32 "
                     "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
                     : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]), "=f"(v[4]), "=f"(v[5]), "=f"(v[6]), "=f"(v[7]),
                       "=f"(v[8]), "=f"(v[9]), "=f"(v[10]), "=f"(v[11]), "=f"(v[12]), "=f"(v[13]), "=f"(v[14]), "=f"(v[15])
                     : "r"(taddr) : "memory");
}
template <int kRegs>
__device__ __forceinline__ void tc_loaded(float (&v)[kRegs])
{
    if constexpr (kRegs == 8)
        asm volatile("tcgen05.wait::ld.sync.aligned;"
                     : "+f"(v[0]), "+f"(v[1]), "+f"(v[2]), "+f"(v[3]), "+f"(v[4]), "+f"(v[5]), "+f"(v[6]), "+f"(v[7]) :: "memory");
    else
        tc_loaded16(v);
}
__device__ __forceinline__ float2 mul2(float2 a, float2 b)
{
    uint64_t x, y, d;
    asm("mov.b64 %0, {%1, %2};" : "=l"(x) : "f"(a.x), "f"(a.y));
    asm("mov.b64 %0, {%1, %2};" : "=l"(y) : "f"(b.x), "f"(b.y));
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(x), "l"(y));
    float2 r;
    asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(d));
    return r;
}
// Four 8 x 8 blocks of 16-bit values to shared memory; lane i has the address of row i % 8 of block i / 8.
__device__ __forceinline__ void store_matrices(unsigned addr, unsigned a, unsigned b, unsigned c, unsigned d)
{
    asm volatile("stmatrix.sync.aligned.m8n8.x4.shared.b16 [%0], {%1, %2, %3, %4};"
                 :: "r"(addr), "r"(a), "r"(b), "r"(c), "r"(d) : "memory");
}

// Two weights as 16-bit high parts and what those leave, as 16-bit low parts.
// fp16 ones are scaled by kGroupWeightScale, against the type's narrow range: a reference lags by 2^7 at most, and small
// weights keep their bits.  Together the parts hold 22 bits (fp16) or 16 (bf16), where the output is rounded to 11 or 8: of 64
// sequences of 4k to 16k tokens with 16 heads, bf16, 0.23 % of the values are not the nearest (0.09 % with 32-bit weights), and the
// error against 64 bits is 1.6593e-3 of the norm either way.
template <typename E>
constexpr float kLatentWeightScale = std::is_same<E, __half>::value ? kGroupWeightScale : 1.f;
template <typename E>
__device__ __forceinline__ void split_weights(float2 w, unsigned &hi, unsigned &lo)
{
    if constexpr (std::is_same<E, __half>::value) {
        w = mul2(w, make_float2(kGroupWeightScale, kGroupWeightScale));
        hi = pack_half2(w.x, w.y);
        const float2 back = __half22float2(*reinterpret_cast<const __half2 *>(&hi));
        lo = pack_half2(w.x - back.x, w.y - back.y);
    } else {
        const __nv_bfloat162 high = __floats2bfloat162_rn(w.x, w.y);
        const float2 back = __bfloat1622float2(high);
        const __nv_bfloat162 low = __floats2bfloat162_rn(w.x - back.x, w.y - back.y);
        hi = *reinterpret_cast<const unsigned *>(&high);
        lo = *reinterpret_cast<const unsigned *>(&low);
    }
}
template <typename E>
__device__ __forceinline__ E latent_round(float x)
{
    if constexpr (std::is_same<E, __half>::value) return __float2half_rn(x);
    else return __float2bfloat16_rn(x);
}
// The new token that query row r belongs to, r / q_heads: (r + 1/2) / q_heads is further from a whole number than 32 bits
// are off, with r < 2^14.
__device__ __forceinline__ int latent_node(int r, float heads_inverse) { return (int)(((float)r + 0.5f) * heads_inverse); }

// Which of the new tokens `at` and at + 8 (negative: positions before them) node `node` of `nodes` sees, by the mask.
__device__ __forceinline__ unsigned latent_sees(const TreeShape &tree, int b, int node, int nodes, int at)
{
    if (node >= nodes) return 0;
    const uint64_t *words = tree.mask + ((int64_t)b * tree.tokens + node) * tree.words;
    auto one = [&](int j) -> unsigned { return j < 0 ? 1u : j < nodes ? (unsigned)(words[j >> 6] >> (j & 63) & 1u) : 0u; };
    return one(at) | one(at + 8) << 1;
}

// Whether none of 8 values is an infinity or a NaN.
template <typename E>
__device__ __forceinline__ bool latent_finite8(const uint4 &x)
{
    if constexpr (std::is_same<E, __half>::value) return finite8(x);
    auto two = [](unsigned w) { return (w & 0x7F80u) != 0x7F80u && (w & 0x7F800000u) != 0x7F800000u; };
    return two(x.x) && two(x.y) && two(x.z) && two(x.w);
}

template <typename E, int L, int N>
__global__ void __launch_bounds__(LatentGeometry<L, N>::kThreads, 1)
latent_attn_kernel(const __grid_constant__ LatentParams p, const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_cache)
{
    using Geo = LatentGeometry<L, N>;
    constexpr int kItems = Geo::kItems, kPanels = Geo::kPanels, kSlots = Geo::kSlots, kRopeSlots = Geo::kRopeSlots;
    constexpr int kSoftmaxWarps = 4;
    constexpr int kWarpCopy = kSoftmaxWarps, kWarpLogits = kWarpCopy + 1, kWarpOutput = kWarpCopy + 2;
    constexpr unsigned kTypes = std::is_same<E, __half>::value ? 0u : 1u << 7 | 1u << 10;      // of A and B in the instruction descriptor
    extern __shared__ unsigned char smem_raw[];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    allow_next_kernel();
    wait_for_previous_kernels();

    const unsigned raw = static_cast<unsigned>(__cvta_generic_to_shared(smem_raw));
    const unsigned base = (raw + 1023u) & ~1023u;
    unsigned char *smem = smem_raw + (base - raw);
    const unsigned rope_smem = base + Geo::kRopeOffset, q_smem = base + Geo::kQOffset, p_smem = base + Geo::kPOffset, misc = base + Geo::kMiscOffset;
    unsigned char *misc_ptr = smem + Geo::kMiscOffset;
    auto entry = [&](int k) -> LatentSegment & { return reinterpret_cast<LatentSegment *>(misc_ptr + kLatSegments)[k & 3]; };
    auto wait_segment = [&](int k) -> bool { return __all_sync(0xffffffffu, tree_wait(misc + kLatBarSegFull + (k & 3) * 8, (k >> 2) & 1)); };
    auto done_segment = [&](int k) {
        __syncwarp();
        if (lane == 0) mbarrier_arrive(misc + kLatBarSegEmpty + (k & 3) * 8);
    };

    LatentFinder finder;               // (of the copying warp)
    finder.plane = blockIdx.x % p.planes;
    finder.team = blockIdx.x / p.planes;
    finder.items = latent_plane_items(p, finder.plane);
    finder.w0 = finder.start = 0;
    if (p.batch > 32) latent_scan(p, misc_ptr, Geo::kThreads, finder.plane, finder.items, finder.team);
    LatentSegment seg;
    if (warp == kWarpLogits) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;"
                     :: "r"(misc + kLatTmemPtr), "n"(Geo::kTmemCols) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    } else if (warp == kWarpCopy && p.batch <= 32) {
        if (lane < 2) asm volatile("prefetch.tensormap [%0];" :: "l"(reinterpret_cast<uint64_t>(lane ? &map_cache : &map_q)) : "memory");
        finder.load(p, lane);
        if (blockIdx.x == 0 && lane < p.batch) {                  // lengths out of range
            int nodes;
            (void)checked_tree(p.tree, p.seq_lens, p.max_seq_len, p.status, lane, true, nodes);
        }
        finder.begin(p, __shfl_sync(0xffffffffu, finder.stop, 31));
        seg = finder.template next<E, L>(p, lane);
    } else if (warp == kWarpOutput && lane == 0) {
        for (int s = 0; s < 12; ++s) {
            mbarrier_init(misc + kLatBarFull + s * 8, 1);
            mbarrier_init(misc + kLatBarEmpty + s * 8, 1);
        }
        for (int s = 0; s < 4; ++s) {
            mbarrier_init(misc + kLatBarRopeFull + s * 8, 1);
            mbarrier_init(misc + kLatBarRopeEmpty + s * 8, 1);
            mbarrier_init(misc + kLatBarSegFull + s * 8, 1);
            mbarrier_init(misc + kLatBarSegEmpty + s * 8, kSoftmaxWarps + 2);     // the two MMA issuers too
        }
        for (int s = 0; s < 2; ++s) {
            mbarrier_init(misc + kLatBarSFull + s * 8, 1);
            mbarrier_init(misc + kLatBarSFree + s * 8, kSoftmaxWarps);
        }
        mbarrier_init(misc + kLatBarPFull, kSoftmaxWarps);
        mbarrier_init(misc + kLatBarPvDone, 1);
        mbarrier_init(misc + kLatBarQFull, 1);
        mbarrier_init(misc + kLatBarQEmpty, 1);
        mbarrier_init_fence();
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const unsigned tmem = *reinterpret_cast<volatile unsigned *>(misc_ptr + kLatTmemPtr);

    if (warp == kWarpCopy) {
        // ================================ copies ================================
        const bool paged = p.block_table != nullptr;
        const int T = p.run_tokens;
        if (p.batch > 32) {
            const int *found = reinterpret_cast<const int *>(misc_ptr + kLatTotal);
            finder.begin(p, found[0]);
            if (finder.tile < finder.end) {
                finder.w0 = found[1];
                finder.start = found[2];
                finder.load(p, lane);
            }
            seg = finder.template next<E, L>(p, lane);
        }
        int g = 0, k = 0;                                 // tiles and segments so far
        bool fine = true;
        // lane i: the physical block of the i-th run of tile j (asked for one tile ahead; bringing the next tile into L2 meanwhile,
        // as the pairs' kernel does, costs 12 % here: 64 sequences of 4k-16k, 16 heads, 159 us against 140)
        auto fetch_ids = [&](const LatentSegment &s, int j) -> int {
            if (!paged) return 0;
            const int start = j * kLatentTile;
            if (j >= s.t1 || lane >= (min(s.len - start, kLatentTile) + T - 1) / T) return -1;
            const int idx = (start + lane * T) / p.block_tokens;
            if (!bounds_ok(idx < p.max_blocks_per_seq, p.status)) return -1;
            return p.block_table[(int64_t)s.b * p.max_blocks_per_seq + idx];
        };
        auto copy_tile = [&](const LatentSegment &s, int j, int phys) -> bool {
            const int start = j * kLatentTile, nb = (min(s.len - start, kLatentTile) + T - 1) / T;
            bool good = lane < nb;
            int row;                                      // (< 2^31 rows: checked by the host)
            if (paged) {
                const bool in_range = phys >= 0 && (int64_t)phys < p.num_phys_blocks;
                if (good && !in_range && p.status) atomicOr(p.status, kFlagBlockRange);
                row = in_range ? phys * p.block_tokens + (start + lane * T) % p.block_tokens : 0;
                good = good && in_range && bounds_ok((int64_t)row + T <= p.cache_rows, p.status);
            } else {
                row = s.b * p.s_max + start;              // rows past the tensor's end read as zeros
            }
            const unsigned fetched = __popc(__ballot_sync(0xffffffffu, good));
            const bool missing = lane < nb && !good;      // a block that cannot be read counts as zeros
            const bool any_missing = __any_sync(0xffffffffu, missing);
            // (lane r + 8 q asks for panel q of run r)
            const int my_row = __shfl_sync(0xffffffffu, row, lane & 7);
            const bool my_good = __shfl_sync(0xffffffffu, (int)good, lane & 7) != 0;
            const unsigned my_at = (lane & 7) * T * 128 + (lane >> 3) * kLatentPanel;
            // One item of `panels` panels into a slot; the slot is free.
            auto copy_item = [&](unsigned slot_offset, unsigned bar, int dim, int panels) {
                if (any_missing) {
                    if (missing) {
                        const uint4 zero = make_uint4(0u, 0u, 0u, 0u);
#pragma unroll 1
                        for (int panel = 0; panel < panels; ++panel)
#pragma unroll 1
                            for (int i = 0; i < T * 8; ++i) *reinterpret_cast<uint4 *>(smem + slot_offset + lane * T * 128 + panel * kLatentPanel + i * 16) = zero;
                        fence_async_proxy();
                    }
                    __syncwarp();
                }
                if (lane == 0) mbarrier_expect_bytes(bar, fetched * (unsigned)(T * 128 * panels));
                __syncwarp();
                if (my_good && lane < 8 * panels) tma_load_2d(base + slot_offset + my_at, &map_cache, dim + (lane >> 3) * 64, my_row, bar);
            };
#pragma unroll 1
            for (int item = 0; item < kItems; ++item) {
                const int n = g * kItems + item, slot = n % kSlots;
                if (n >= kSlots && !__all_sync(0xffffffffu, tree_wait(misc + kLatBarEmpty + slot * 8, (n / kSlots - 1) & 1))) return false;
                copy_item(slot * kLatentItem, misc + kLatBarFull + slot * 8, item * 128, 2);
            }
            const int slot = g % kRopeSlots;
            if (g >= kRopeSlots && !__all_sync(0xffffffffu, tree_wait(misc + kLatBarRopeEmpty + slot * 8, (g / kRopeSlots - 1) & 1))) return false;
            copy_item(Geo::kRopeOffset + slot * kLatentPanel, misc + kLatBarRopeFull + slot * 8, L, 1);
            return true;
        };
        auto announce = [&](const LatentSegment &s, int n) -> bool {
            if (n >= 4 && !__all_sync(0xffffffffu, tree_wait(misc + kLatBarSegEmpty + (n & 3) * 8, ((n >> 2) - 1) & 1))) return false;
            if (lane == 0) {
                entry(n) = s;
                mbarrier_arrive(misc + kLatBarSegFull + (n & 3) * 8);
            }
            return true;
        };
        // A segment is found while the copies of the one before run.
        (void)announce(seg, 0);
        int ids = seg.b >= 0 ? fetch_ids(seg, seg.t0) : -1;
        bool asked_q = false;
        for (; fine && seg.b >= 0; ++k) {
            LatentSegment after = seg;                    // segment k + 1
            int ids_after = -1;
            for (int j = seg.t0; j < seg.t1 && fine; ++j) {
                if (j == seg.t0) {
                    // the query rows wait for the last segment's logits
                    if (k >= 1) fine = __all_sync(0xffffffffu, tree_wait(misc + kLatBarQEmpty, (k - 1) & 1));
                    if (!fine) break;
                    if (lane == 0) mbarrier_expect_bytes(misc + kLatBarQFull, (unsigned)Geo::kQBytes);
                    __syncwarp();
                    if (lane <= kPanels)                      // (rows behind the sequence's last are zeros)
                        tma_load_3d(q_smem + lane * Geo::kQPanel, &map_q, lane * 64, seg.row0, seg.b, misc + kLatBarQFull);
                    asked_q = true;
                    __syncwarp();
                }
                const int now = ids;
                ids = fetch_ids(seg, j + 1);
                fine = copy_tile(seg, j, now);
                if (fine) ++g;
                if (j > seg.t0 || !fine) continue;
                after = finder.template next<E, L>(p, lane);
                fine = announce(after, k + 1);
                if (after.b >= 0) ids_after = fetch_ids(after, after.t0);
            }
            if (!fine) break;
            asked_q = false;
            seg = after;
            ids = ids_after;
        }
        if (!fine) {
            if (lane == 0 && p.status) atomicOr(p.status, kFlagCopyTimeout);
            // copies in flight must land (or be given up, bounded) before shared memory is handed on; the tile that was
            // given up may have some of its items
            for (int n = max((g + 1) * kItems - kSlots, 0); n < (g + 1) * kItems; ++n)
                (void)tree_wait(misc + kLatBarFull + (n % kSlots) * 8, (n / kSlots) & 1);
            for (int n = max(g + 1 - kRopeSlots, 0); n < g + 1; ++n)
                (void)tree_wait(misc + kLatBarRopeFull + (n % kRopeSlots) * 8, (n / kRopeSlots) & 1);
            if (asked_q) (void)tree_wait(misc + kLatBarQFull, k & 1);
        }
    } else if (warp == kWarpLogits) {
        // ================================ logit MMAs ================================
        constexpr unsigned idesc = umma_idesc(64, N, 0, 0) | kTypes;   // tile and query rows K-major
        const uint64_t q_desc = umma_desc(q_smem, 16, 1024, 2);
        bool fine = true;
        int g = 0;
        for (int k = 0; fine; ++k) {
            fine = wait_segment(k);
            if (!fine) break;
            const int b = entry(k).b, t0 = entry(k).t0, t1 = entry(k).t1;
            done_segment(k);
            if (b < 0) break;
            fine = __all_sync(0xffffffffu, tree_wait(misc + kLatBarQFull, k & 1));
            for (int j = t0; j < t1 && fine; ++j, ++g) {
                const int buf = g & 1;
                if (g >= 2) fine = __all_sync(0xffffffffu, tree_wait(misc + kLatBarSFree + buf * 8, ((g >> 1) - 1) & 1));
                // rows of 128 bytes per panel, 8-row groups 1024 bytes apart; a k-step of 16 dims is 32 bytes along the row
#pragma unroll
                for (int item = 0; item <= kItems; ++item) {
                    if (!fine) break;
                    const bool rope = item == kItems;
                    const int n = rope ? g : g * kItems + item, slots = rope ? kRopeSlots : kSlots, slot = n % slots;
                    fine = __all_sync(0xffffffffu, tree_wait(misc + (rope ? kLatBarRopeFull : kLatBarFull) + slot * 8, (n / slots) & 1));
                    if (!fine) break;
                    tc_fence_after();
                    const uint64_t tile_desc = umma_desc(rope ? rope_smem + slot * kLatentPanel : base + slot * kLatentItem, 16, 1024, 2);
                    if (elect_one()) {
#pragma unroll
                        for (int ks = 0; ks < (rope ? 4 : 8); ++ks)
                            tc_mma_f16(tmem + buf * N, tile_desc + (uint64_t)(((ks >> 2) * kLatentPanel + (ks & 3) * 32) >> 4),
                                       q_desc + (uint64_t)(((item * 2 + (ks >> 2)) * Geo::kQPanel + (ks & 3) * 32) >> 4), idesc,
                                       item > 0 || ks > 0);
                        if (rope) {
                            tc_commit(misc + kLatBarRopeEmpty + slot * 8);
                            tc_commit(misc + kLatBarSFull + buf * 8);
                            if (j + 1 == t1) tc_commit(misc + kLatBarQEmpty);
                        }
                    }
                    __syncwarp();
                }
            }
        }
        if (!fine && lane == 0 && p.status) atomicOr(p.status, kFlagCopyTimeout);
    } else if (warp == kWarpOutput) {
        // ================================ output MMAs ================================
        constexpr unsigned idesc = umma_idesc(128, Geo::kAccCols, 1, 1) | kTypes;   // tile and weights MN-major
        // Weights: 8-column blocks of [64 tokens][16 bytes], 1024 bytes apart; 8-token groups 128 bytes apart; a k-step is
        // 16 tokens = 256 bytes.  The low parts lie behind the high ones.
        const uint64_t p_desc = umma_desc(p_smem, 128, 1024, 0);
        bool fine = true;
        int g = 0;
        for (int k = 0; fine; ++k) {
            fine = wait_segment(k);
            if (!fine) break;
            const int b = entry(k).b, t0 = entry(k).t0, t1 = entry(k).t1;
            done_segment(k);
            if (b < 0) break;
            for (int j = t0; j < t1 && fine; ++j, ++g) {
                fine = __all_sync(0xffffffffu, tree_wait(misc + kLatBarPFull, g & 1));
#pragma unroll
                for (int item = 0; item < kItems; ++item) {
                    if (!fine) break;
                    const int n = g * kItems + item, slot = n % kSlots;
                    fine = __all_sync(0xffffffffu, tree_wait(misc + kLatBarFull + slot * 8, (n / kSlots) & 1));
                    if (!fine) break;
                    tc_fence_after();
                    // the tile read MN-major (M = 128 dims): its 64-dim panels kLatentPanel apart, 8-token groups 1024
                    // bytes apart; a k-step is 16 tokens = 2048 bytes
                    const uint64_t v_desc = umma_desc(base + slot * kLatentItem, kLatentPanel, 1024, 2);
                    if (elect_one()) {
                        const unsigned acc = tmem + Geo::kOColumn + item * Geo::kAccCols;
#pragma unroll
                        for (int ks = 0; ks < 4; ++ks)
                            tc_mma_f16(acc, v_desc + (uint64_t)((ks * 2048) >> 4), p_desc + (uint64_t)((ks * 256) >> 4), idesc, j > t0 || ks > 0);
                        tc_commit(misc + kLatBarEmpty + slot * 8);
                        if (item + 1 == kItems) tc_commit(misc + kLatBarPvDone);
                    }
                    __syncwarp();
                }
            }
        }
        if (!fine && lane == 0 && p.status) atomicOr(p.status, kFlagCopyTimeout);
    } else {
        // ================================ softmax and epilogue ================================
        const int quarter = warp;                                     // this warp's tokens: 16 of the tile
        const int t = threadIdx.x & 127;
        const int token = quarter * 16 + (lane >> 2), column = 2 * (lane & 3);        // this thread's tokens: token, token + 8
        const unsigned lanes = tmem + ((unsigned)(quarter * 32) << 16);
        constexpr int kPer = N / 8;                                   // pairs of columns of a thread
        float *by_warp = reinterpret_cast<float *>(misc_ptr + kLatMiscBytes);        // [N][4]: a row's maxima, or sums, by warp
        float *offsets = by_warp + N * 4;                             // [N]: the rows' references (negated) as they were last moved
        const float scale = p.scale_log2e, sign = copysignf(1.f, scale), heads_inverse = 1.f / (float)p.q_heads;
        bool fine = true;
        int g = 0;
        for (int k = 0;; ++k) {
            // (one decision for all: their barriers have to stay in step)
            if (group_any(1, !wait_segment(k) || !fine)) {
                fine = false;
                break;
            }
            const LatentSegment &seg = entry(k);
            if (seg.b < 0) break;
            const int len = seg.len, nodes = seg.nodes, prefix = seg.prefix(), t0 = seg.t0, t1 = seg.t1, row0 = seg.row0;
            // [pair of columns][one of the pair]: the negated reference, a logit before the scale; sums of this thread's tokens
            float2 offset[kPer], l[kPer];
#pragma unroll
            for (int j = 0; j < kPer; ++j) {
                offset[j] = make_float2(-kMinusHuge * sign, -kMinusHuge * sign);
                l[j] = make_float2(0.f, 0.f);
            }
            for (int j = t0; j < t1; ++j, ++g) {
                const int buf = g & 1, start = j * kLatentTile;
                const unsigned logits = lanes + buf * N;
                const bool masked = start + kLatentTile > prefix;     // uniform
                unsigned hidden = 0;                                  // bit 4 i + 2 u + c: column c of pair i does not see token u
                if (masked) {
                    const int at = start + token - prefix;            // the first token as a new one; the second is at + 8
#pragma unroll 1
                    for (int i = 0; i < 2 * kPer; ++i) {              // column i % 2 of pair i / 2
                        const int node = latent_node(row0 + 8 * (i >> 1) + column + (i & 1), heads_inverse);
                        unsigned sees = (at <= node ? 1u : 0u) | (at + 8 <= node ? 2u : 0u);
                        if (p.tree.mask != nullptr) sees = latent_sees(p.tree, seg.b, node, nodes, at);
                        if (node >= nodes) sees = 0;
                        hidden |= ((~sees & 1u) | (~sees & 2u) << 1) << (4 * (i >> 1) + (i & 1));
                    }
                }
                if (fine) fine = tree_wait(misc + kLatBarSFull + buf * 8, (g >> 1) & 1);
                fine = __all_sync(0xffffffffu, fine);
                tc_fence_after();
                float x[4 * kPer], e[4 * kPer];
                tc_issue_load_16lanes(x, logits);
                // Exponents of the weights against the references; where one is too large the references move and they
                // are computed again.
                for (int attempt = 0;; ++attempt) {
                    tc_loaded(x);
                    float most = -INFINITY, most_odd = -INFINITY;
#pragma unroll
                    for (int i = 0; i < 2 * kPer; ++i) {              // pair i / 2 of token i % 2
                        const float2 y = mul2(add2(make_float2(x[2 * i], x[2 * i + 1]), offset[i / 2]), make_float2(scale, scale));
                        e[2 * i] = y.x;
                        e[2 * i + 1] = y.y;
                    }
                    if (masked) {
#pragma unroll
                        for (int i = 0; i < 4 * kPer; ++i)
                            if (hidden >> i & 1u) e[i] = -INFINITY;
                    }
#pragma unroll
                    for (int i = 0; i < 4 * kPer; i += 4) {
                        most = max3(most, e[i], e[i + 1]);
                        most_odd = max3(most_odd, e[i + 2], e[i + 3]);
                    }
                    if (attempt > 0 || !group_any(1, fmaxf(most, most_odd) > kGroupLag)) break;
                    // ---- some row's reference moves (rare after a segment's first tile) ----
                    if (j > t0) {                                     // the accumulators hold the tiles before this one
                        if (fine) fine = tree_wait(misc + kLatBarPvDone, (g - 1) & 1);
                        fine = __all_sync(0xffffffffu, fine);
                        tc_fence_after();
                    }
#pragma unroll
                    for (int i = 0; i < kPer; ++i) {
                        float top[2];
#pragma unroll
                        for (int c = 0; c < 2; ++c) {
                            const float a = hidden >> (4 * i + c) & 1u ? -INFINITY : x[4 * i + c] * sign;
                            const float b = hidden >> (4 * i + 2 + c) & 1u ? -INFINITY : x[4 * i + 2 + c] * sign;
                            top[c] = fmaxf(a, b);
#pragma unroll
                            for (int o = 4; o < 32; o <<= 1) top[c] = fmaxf(top[c], __shfl_xor_sync(0xffffffffu, top[c], o));
                            if (lane < 4) by_warp[(8 * i + column + c) * 4 + quarter] = top[c];
                        }
                    }
                    group_sync(2);
                    float2 alpha[kPer];                               // 2^(old - new reference)
#pragma unroll
                    for (int i = 0; i < kPer; ++i) {
#pragma unroll
                        for (int c = 0; c < 2; ++c) {
                            const float4 tops = *reinterpret_cast<const float4 *>(by_warp + (8 * i + column + c) * 4);
                            const float top = max3(fmaxf(tops.x, tops.y), tops.z, tops.w);
                            float &off = c ? offset[i].y : offset[i].x, &sum = c ? l[i].y : l[i].x, &factor = c ? alpha[i].y : alpha[i].x;
                            factor = 1.f;
                            const float moved = -top * sign, rise = (off - moved) * scale;
                            if (rise > kGroupLag) {
                                factor = fast_exp2(-rise);
                                off = moved;
                                if (quarter == 0 && lane < 4) offsets[8 * i + column + c] = off;
                            }
                            sum *= factor;
                        }
                    }
                    group_sync(2);                                    // the maxima have been read
                    if (j > t0) {
                        if (quarter == 0 && lane < 4) {
#pragma unroll
                            for (int i = 0; i < kPer; ++i) {
                                by_warp[(8 * i + column) * 4] = alpha[i].x;
                                by_warp[(8 * i + column + 1) * 4] = alpha[i].y;
                            }
                        }
                        group_sync(2);
#pragma unroll 1
                        for (int acc = 0; acc < kItems; ++acc) {
#pragma unroll 1
                            for (int part = 0; part < 2; ++part) {          // high and low columns
#pragma unroll 1
                                for (int c0 = 0; c0 < N; c0 += 16) {
                                    const unsigned at = lanes + Geo::kOColumn + acc * Geo::kAccCols + part * N + c0;
                                    float o[16];
                                    tc_issue_load16(o, at);
                                    tc_loaded16(o);
#pragma unroll
                                    for (int c = 0; c < 16; ++c) o[c] *= by_warp[(c0 + c) * 4];
                                    tc_store16(at, o);
                                }
                            }
                        }
                        group_sync(2);                                // the factors have been read
                    }
                    tc_issue_load_16lanes(x, logits);
                }
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbarrier_arrive(misc + kLatBarSFree + buf * 8);
                unsigned hi[2 * kPer], lo[2 * kPer];                  // pair i / 2 of token i % 2
#pragma unroll
                for (int i = 0; i < 2 * kPer; ++i) {
                    const float2 w = make_float2(fast_exp2(e[2 * i]), fast_exp2(e[2 * i + 1]));
                    l[i / 2] = add2(l[i / 2], w);
                    split_weights<E>(w, hi[i], lo[i]);
                }
                if (g > 0 && fine) fine = tree_wait(misc + kLatBarPvDone, (g - 1) & 1);        // the last tile's MMAs have read the weights
                if (masked) {
                    // Value rows behind the sequence get weight 0 but may hold anything, and 0 x NaN is NaN: they are
                    // cleared.  So are new tokens' rows that are not finite: a row that sees one has a logit that is
                    // not finite (its values are part of its key), which makes the row NaN, or leaves the token out, without them.
                    // A row is L / 8 chunks of 16 bytes, a lane's are those of panel lane / 8 and of the panel four further on.
                    const int first = quarter * 16, last = first + 16;
                    if (start + last > prefix) {
                        // (the logits have read the tile: it has landed)
                        const int item = g * kItems + min(lane, kItems - 1);
                        if (fine) fine = tree_wait(misc + kLatBarFull + item % kSlots * 8, (item / kSlots) & 1);
                        __syncwarp();
                        unsigned char *chunks[kPanels / 4];
#pragma unroll
                        for (int i = 0; i < kPanels / 4; ++i)
                            chunks[i] = smem + (g * kItems + (lane >> 4) + 2 * i) % kSlots * kLatentItem + (lane >> 3 & 1) * kLatentPanel + (lane & 7) * 16;
#pragma unroll 1
                        for (int r = max(first, prefix - start); r < last; ++r) {
                            if (start + r < len) {
                                bool bad = false;
#pragma unroll
                                for (int i = 0; i < kPanels / 4; ++i) bad = bad | !latent_finite8<E>(*reinterpret_cast<const uint4 *>(chunks[i] + r * 128));
                                if (!__any_sync(0xffffffffu, bad)) continue;
                            }
#pragma unroll
                            for (int i = 0; i < kPanels / 4; ++i) *reinterpret_cast<uint4 *>(chunks[i] + r * 128) = make_uint4(0u, 0u, 0u, 0u);
                        }
                    }
                }
                // Lane i has the address of token row i % 8 of block i / 8: tokens 0-7 and 8-15 of two blocks of 8 columns.
                const unsigned to = p_smem + (lane >> 4) * 1024 + (quarter * 16 + (lane >> 3 & 1) * 8 + (lane & 7)) * 16;
#pragma unroll
                for (int i = 0; i < kPer; i += 2) {
                    store_matrices(to + i * 1024, hi[2 * i], hi[2 * i + 1], hi[2 * i + 2], hi[2 * i + 3]);
                    store_matrices(to + i * 1024 + Geo::kPPart, lo[2 * i], lo[2 * i + 1], lo[2 * i + 2], lo[2 * i + 3]);
                }
                fence_async_proxy();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbarrier_arrive(misc + kLatBarPFull);
            }
            // ---- the segment's end: row sums, then the accumulators divided by them; thread t has dim t of each ----
#pragma unroll
            for (int i = 0; i < kPer; ++i) {
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    float sum = c ? l[i].y : l[i].x;
#pragma unroll
                    for (int o = 4; o < 32; o <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
                    if (lane < 4) by_warp[(8 * i + column + c) * 4 + quarter] = sum;
                }
            }
            group_sync(2);
            const bool whole = seg.whole();
            if (t < N) {
                // one thread per row: its sum's inverse (0: a row of zeros) and its log-sum-exp
                const int r = t;
                const float4 sums = *reinterpret_cast<const float4 *>(by_warp + r * 4);
                const float total = (sums.x + sums.y) + (sums.z + sums.w);
                const bool empty = r >= seg.rows || (seg.row0 + r) / p.q_heads >= nodes || total == 0.f;     // (a NaN sum is not an empty row's)
                if (r < seg.rows && fine && seg.lse)
                    seg.lse[r] = empty ? (whole ? -INFINITY : kMinusHuge) : fmaf(-offsets[r], p.scale, logf(total));
                by_warp[r * 4] = empty ? 0.f : __fdividef(1.f / kLatentWeightScale<E>, total);
            }
            if (fine) fine = tree_wait(misc + kLatBarPvDone, (g - 1) & 1);
            fine = __all_sync(0xffffffffu, fine);
            tc_fence_after();
            group_sync(2);
#pragma unroll 1
            for (int block = 0; block < N / 16 * kItems; ++block) {
                const int first = block / kItems * 16, acc = block % kItems, d = acc * 128 + t;
                const unsigned at = lanes + Geo::kOColumn + acc * Geo::kAccCols + first;
                float o[16];
                tc_issue_load16(o, at);
                float low[16];
                tc_issue_load16(low, at + N);
                tc_loaded16(o);
                tc_loaded16(low);
#pragma unroll
                for (int i = 0; i < 16; ++i) o[i] += low[i];
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const float inverse = by_warp[(first + i) * 4];
                    o[i] = inverse == 0.f ? 0.f : o[i] * inverse;     // (an empty row's accumulator may hold anything)
                }
                const int rows = fine ? seg.rows - first : 0;
                if (whole) {
                    E *out = static_cast<E *>(seg.out) + first * L + d;
#pragma unroll
                    for (int i = 0; i < 16; ++i)
                        if (i < rows) out[i * L] = latent_round<E>(o[i]);
                } else {
                    float *out = static_cast<float *>(seg.out) + first * L + d;
#pragma unroll
                    for (int i = 0; i < 16; ++i)
                        if (i < rows) out[i * L] = o[i];
                }
                __syncwarp();
            }
            tc_fence_before();                                        // the accumulators have been read: the next tile may overwrite them
            group_sync(2);                                            // so have the rows' numbers
            done_segment(k);
        }
        if (!fine && lane == 0 && p.status) atomicOr(p.status, kFlagCopyTimeout);
    }

    // ---- teardown: everyone is done with tensor memory before it is released ----
    tc_fence_before();
    __syncthreads();
    if (warp == kWarpLogits) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" :: "r"(tmem), "n"(Geo::kTmemCols) : "memory");
    }
}

// Joins the partial results of the items that more than one share has a part of, and zeroes the rows of sequences
// without work.  A warp takes kDims dims of one row: the kernel is a chain of loads (the item's shares, their
// log-sum-exps, the partials), so few rows are cut into 128 dims each, whose partials are few rounds of loads, while
// whole rows leave the fewest warps where there are more than fit the GPU at once.
constexpr int kLatentMergeThreads = 256;

template <typename E, int L, int kDims>
__global__ void __launch_bounds__(kLatentMergeThreads)
latent_merge_kernel(const LatentParams p, int row_parts)
{
    constexpr int kPieces = L / kDims, kRows = kLatentMergeThreads / 32 / kPieces;      // warps of a row, rows of a block
    constexpr int kVecs = kDims / 128, kDeep = 8 / kVecs;             // a lane's dims: kVecs runs of four; partials in flight
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int part = blockIdx.x % row_parts, item = blockIdx.x / row_parts;           // (sequence, row block)
    const int b = item / p.row_blocks, rb = item - b * p.row_blocks;
    const int r = part * kRows + warp / kPieces, row = rb * p.block_rows + r, d = warp % kPieces * kDims + lane * 4;
    allow_next_kernel();
    wait_for_previous_kernels();
    int nodes;
    const int2 shares = p.item_shares[item];
    const int len = checked_tree(p.tree, p.seq_lens, p.max_seq_len, nullptr, b, false, nodes);
    const int c0 = shares.x, n = latent_tiles(p, len, nodes) > 0 ? shares.y - c0 + 1 : 0;
    if (n == 1) return;                                               // one share had it all: the result is written
    if (r >= p.block_rows || row >= p.rows) return;
    const int64_t out_row = (int64_t)b * p.rows + row;
    // (the item's start went to its block's second slot, all else to the first one)
    auto slot_row = [&](int i) -> int64_t { return (int64_t)(2 * (rb % p.planes + (c0 + i) * p.planes) + (i == 0 ? 1 : 0)) * p.block_rows + r; };
    float top = kMinusHuge, total = 0.f;
    bool any_nan = false;
    float first_lse = kMinusHuge;                                     // of the first 32 partials, a lane each
    for (int i = lane; i < n; i += 32) {
        const float lse = p.part_lse[slot_row(i)];
        if (i < 32) first_lse = lse;
        top = fmaxf(top, lse);
        any_nan = any_nan || lse != lse;
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
    const bool empty = !(top > kMinusHuge) && !__any_sync(0xffffffffu, any_nan);
    float4 acc[kVecs];
#pragma unroll
    for (int v = 0; v < kVecs; ++v) acc[v] = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int i0 = 0; i0 < n && !empty; i0 += 32) {
        const float lse = i0 == 0 ? first_lse : i0 + lane < n ? p.part_lse[slot_row(i0 + lane)] : kMinusHuge;
        const float mine = i0 + lane < n ? fast_exp2((lse - top) * 1.44269504088896340736f) : 0.f;
        const int here = min(32, n - i0);
        for (int i = 0; i < here; i += kDeep) {
            float4 x[kDeep][kVecs];
#pragma unroll
            for (int u = 0; u < kDeep; ++u) {
#pragma unroll
                for (int v = 0; v < kVecs; ++v)
                    x[u][v] = i + u < here ? *reinterpret_cast<const float4 *>(p.part_o + slot_row(i0 + i + u) * L + d + v * 128) : make_float4(0.f, 0.f, 0.f, 0.f);
            }
#pragma unroll
            for (int u = 0; u < kDeep; ++u) {
                const float w = __shfl_sync(0xffffffffu, mine, (i + u) & 31);
                if (i + u < here) {
                    total += w;
#pragma unroll
                    for (int v = 0; v < kVecs; ++v) {
                        acc[v].x = fmaf(w, x[u][v].x, acc[v].x);
                        acc[v].y = fmaf(w, x[u][v].y, acc[v].y);
                        acc[v].z = fmaf(w, x[u][v].z, acc[v].z);
                        acc[v].w = fmaf(w, x[u][v].w, acc[v].w);
                    }
                }
            }
        }
    }
    const float inverse = empty ? 0.f : 1.f / total;
#pragma unroll
    for (int v = 0; v < kVecs; ++v) {
        const E four[4] = {latent_round<E>(empty ? 0.f : acc[v].x * inverse), latent_round<E>(empty ? 0.f : acc[v].y * inverse),
                           latent_round<E>(empty ? 0.f : acc[v].z * inverse), latent_round<E>(empty ? 0.f : acc[v].w * inverse)};
        *reinterpret_cast<uint2 *>(static_cast<E *>(p.out) + out_row * L + d + v * 128) = *reinterpret_cast<const uint2 *>(four);
    }
    if (p.lse && d == 0) p.lse[out_row] = empty ? -INFINITY : top + logf(total);
}

}  // namespace instinfer
