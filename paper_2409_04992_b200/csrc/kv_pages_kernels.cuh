// Bookkeeping of a shared, paged KV cache for sm_100a: keeping the accepted path of a draft tree,
// and forking, resizing (with copy on write) and defragmenting the sequences' blocks.
//
// The state of a pool is one reference count per block (how many sequences' tables list it; 0 =
// free); there is no free list, so nothing depends on the order of earlier calls: an allocation
// takes the lowest free ids.  What moves between pages is a bit copy bound by HBM; what is decided
// (who gets which block) is a few thousand integers and bound by latency, so one thread-block
// cluster decides it in one launch, and a second launch over the whole GPU moves the pages of all
// layers from the list that the first has left in the workspace.
//
// Measured: keeping 7 of 64 nodes of 16 sequences x 40 heads x 40 layers 29.5 us, 5.3 TB/s read and written; 48 forks of
// 16 sequences, their growth with the copies of the shared last blocks in 16 layers, and their release 182 us, 5.5
// TB/s; a defragmentation that moves 3 GB 507 us, 6.0 TB/s.  The smallest calls: keeping a path in one layer 8.9 us, of
// which the GPU works 2.4 (in a graph), the rest is the host's call; a small defragmentation 11.7 us, of which the
// GPU's two launches take 10.4; four forks, their growth and release, five launches, 27.3 us and 21.2 on the GPU.
#pragma once

#include <cooperative_groups.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "tree_common.cuh"

namespace instinfer {

constexpr int kFlagPool = 32;
constexpr int kMaxLayers = 128;          // INSTINFER_MAX_LAYERS: the pointers travel as kernel parameters

struct LayerCaches {
    uint4 *k[kMaxLayers];
    uint4 *v[kMaxLayers];
};

// ---- keeping a path --------------------------------------------------------------------------
struct KeepPathParams {
    const int32_t *path;          // [batch, tree_tokens]
    const int32_t *path_lens;
    const int32_t *tree_lens;     // nullable: tree_tokens each
    const int32_t *seq_lens;
    int32_t *new_lens;
    const int32_t *block_table;   // nullptr: contiguous
    int32_t *status;
    int64_t num_phys_blocks;
    int32_t batch, tree_tokens, heads, s_max, block_tokens, max_blocks_per_seq;
    int32_t segs_per_row;
    int32_t column_blocks;        // thread blocks that share the columns of one (sequence, layer)
    int64_t cache_rows;
};

constexpr int kKeepThreads = 256;
constexpr int kKeepRows = 4;             // rows whose K and V loads are in flight together per thread

// grid: column blocks, fastest, of every (layer, sequence).  Node path[i] of the tree moves from position prefix +
// path[i] to prefix + i.  A path ascends, so path[i] >= i and a row written is never read later:
// each thread takes its 16-byte column of one head through the rows in order, kKeepRows at a time
// (all loads of a step come before its stores), and no thread touches another's column.
__global__ void __launch_bounds__(kKeepThreads)
kv_keep_path_kernel(const KeepPathParams p, const __grid_constant__ LayerCaches caches)
{
    __shared__ int64_t src_row[kMaxTreeTokens], dst_row[kMaxTreeTokens];   // of head 0; -1: not readable
    __shared__ int moves;
    const int part = blockIdx.x % p.column_blocks, rest = blockIdx.x / p.column_blocks;
    const int layer = rest / p.batch, b = rest - layer * p.batch, t = threadIdx.x;
    const bool first = part == 0 && layer == 0;
    if (t == 0) moves = 0;
    asm volatile("griddepcontrol.launch_dependents;");
    asm volatile("griddepcontrol.wait;" ::: "memory");

    const int len = p.seq_lens[b];
    const int nodes = p.tree_lens ? p.tree_lens[b] : p.tree_tokens;
    const int kept = p.path_lens[b];
    const int64_t capacity = p.block_table ? (int64_t)p.max_blocks_per_seq * p.block_tokens : (int64_t)p.s_max;
    const bool len_ok = len >= 0 && len <= capacity;
    bool fine = len_ok && nodes >= 0 && nodes <= p.tree_tokens && nodes <= len && kept >= 0 && kept <= nodes;
    int mine = -1;
    if (fine && t < kept) {
        mine = p.path[(int64_t)b * p.tree_tokens + t];
        const int before = t > 0 ? p.path[(int64_t)b * p.tree_tokens + t - 1] : -1;
        fine = mine > before && mine < nodes;
    }
    // an inactive slot (length 0) is left alone without a flag
    if (__syncthreads_or(!fine)) {
        if (first && t == 0) {
            p.new_lens[b] = len;
            if (len != 0 && p.status) atomicOr(p.status, len_ok ? kFlagTreeRange : kFlagSeqLenRange);
        }
        return;
    }
    const int prefix = len - nodes;
    if (first && t == 0) p.new_lens[b] = prefix + kept;
    const int head_stride = p.block_table ? p.block_tokens : p.s_max;     // rows from one head to the next
    auto row_of = [&](int pos) -> int64_t {
        if (!p.block_table) return (int64_t)b * p.heads * p.s_max + pos;
        const int phys = p.block_table[(int64_t)b * p.max_blocks_per_seq + pos / p.block_tokens];
        if (phys < 0 || (int64_t)phys >= p.num_phys_blocks) {
            if (first && p.status) atomicOr(p.status, kFlagBlockRange);
            return -1;
        }
        return (int64_t)phys * p.heads * p.block_tokens + pos % p.block_tokens;
    };
    if (t < kept && mine != t) {                              // (a path ascends: from its first move on all rows move)
        src_row[t] = row_of(prefix + mine);
        dst_row[t] = row_of(prefix + t);
        atomicAdd(&moves, 1);
    }
    __syncthreads();
    const int begin = kept - moves;
    if (moves == 0) return;
    const int column = part * kKeepThreads + t;               // (head, segment)
    if (column >= p.heads * p.segs_per_row) return;
    const int h = column / p.segs_per_row, seg = column - h * p.segs_per_row;
    const int64_t shift = (int64_t)h * head_stride;
    uint4 *kc = caches.k[layer], *vc = caches.v[layer];
    for (int i0 = begin; i0 < kept; i0 += kKeepRows) {
        uint4 k[kKeepRows], v[kKeepRows];
        bool move[kKeepRows];
#pragma unroll
        for (int u = 0; u < kKeepRows; ++u) {
            const int i = i0 + u;
            move[u] = i < kept && src_row[i] >= 0 && dst_row[i] >= 0;
            if (move[u]) {
                const int64_t s = src_row[i] + shift, d = dst_row[i] + shift;
                move[u] = bounds_ok(s >= 0 && s < p.cache_rows && d >= 0 && d < p.cache_rows, p.status);
                if (move[u]) {
                    k[u] = kc[s * p.segs_per_row + seg];
                    v[u] = vc[s * p.segs_per_row + seg];
                }
            }
        }
#pragma unroll
        for (int u = 0; u < kKeepRows; ++u) {
            if (!move[u]) continue;
            const int64_t d = dst_row[i0 + u] + shift;
            kc[d * p.segs_per_row + seg] = k[u];
            vc[d * p.segs_per_row + seg] = v[u];
        }
    }
}

// ---- forking ---------------------------------------------------------------------------------
struct ForkParams {
    int32_t *block_table;
    int32_t *block_refs;
    int32_t *seq_lens;
    const int32_t *src;
    const int32_t *dst;
    int32_t *status;
    int64_t num_phys_blocks;
    int32_t n_forks, batch, block_tokens, max_blocks_per_seq;
};

constexpr int kForkThreads = 256;

// One block per fork.  A destination listed twice takes the first fork only, and a source may not
// be a destination of the same call, so no block reads what another one writes.
__global__ void __launch_bounds__(kForkThreads)
kv_fork_kernel(const ForkParams p)
{
    asm volatile("griddepcontrol.launch_dependents;");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int i = blockIdx.x;
    const int src = p.src[i], dst = p.dst[i];
    bool bad = src < 0 || src >= p.batch || dst < 0 || dst >= p.batch;
    for (int j = threadIdx.x; j < p.n_forks; j += kForkThreads)
        bad = bad || (j < i && p.dst[j] == dst) || p.dst[j] == src;
    if (__syncthreads_or(bad)) {
        if (threadIdx.x == 0 && p.status) atomicOr(p.status, kFlagPool);
        return;
    }
    const int len = p.seq_lens[src];
    if (len < 0 || (int64_t)len > (int64_t)p.max_blocks_per_seq * p.block_tokens || p.seq_lens[dst] != 0) {
        if (threadIdx.x == 0 && p.status) atomicOr(p.status, kFlagSeqLenRange);
        return;
    }
    __syncthreads();                                          // every thread has read the lengths
    const int held = (int)(((int64_t)len + p.block_tokens - 1) / p.block_tokens);
    const int32_t *from = p.block_table + (int64_t)src * p.max_blocks_per_seq;
    int32_t *to = p.block_table + (int64_t)dst * p.max_blocks_per_seq;
    for (int e = threadIdx.x; e < held; e += kForkThreads) {
        const int id = from[e];
        to[e] = id;
        if (id < 0 || (int64_t)id >= p.num_phys_blocks) {
            if (p.status) atomicOr(p.status, kFlagBlockRange);
        } else if (atomicAdd(p.block_refs + id, 1) <= 0 && p.status) {
            atomicOr(p.status, kFlagPool);                    // a listed block that counted as free
        }
    }
    if (threadIdx.x == 0) p.seq_lens[dst] = len;
}

// ---- deciding a resize -----------------------------------------------------------------------
// Pages to move: pages[2 i] -> pages[2 i + 1], i < *count.
struct PageList {
    int32_t *count;
    int32_t *pages;
};

struct ResizeParams {
    int32_t *block_table;
    int32_t *block_refs;
    const int32_t *seq_lens;
    const int32_t *want_lens;
    int32_t *new_lens;            // may be seq_lens itself
    int32_t *status;
    int64_t num_phys_blocks;
    int32_t batch, block_tokens, max_blocks_per_seq;
    int32_t *counts;              // [batch] blocks that each sequence asks for, with kCopyBit (the first is a copy) or kKeepBit
    int32_t *slices;              // [kPlanCtas] free blocks in each block's range
    PageList list;
};

constexpr int kPlanCtas = 8;             // one portable cluster
constexpr int kPlanThreads = 512;
constexpr int kCopyBit = 1 << 30;
constexpr int kKeepBit = 1 << 29;        // the sequence keeps a block that others leave: it is served only after them
constexpr int kMaxPlanBatch = 8192;      // 16 bytes of shared memory per sequence

// Inclusive sum over the block's threads of a pair of counts; *total = the block's sums.
__device__ __forceinline__ int2 plan_scan(int2 v, int2 *warp_sums, int2 *total)
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int x = __shfl_up_sync(0xffffffffu, v.x, o), y = __shfl_up_sync(0xffffffffu, v.y, o);
        if (lane >= o) {
            v.x += x;
            v.y += y;
        }
    }
    __syncthreads();                                          // warp_sums is free again
    if (lane == 31) warp_sums[warp] = v;
    __syncthreads();
    int2 before = make_int2(0, 0), all = make_int2(0, 0);
#pragma unroll
    for (int w = 0; w < kPlanThreads / 32; ++w) {
        const int2 s = warp_sums[w];
        if (w < warp) {
            before.x += s.x;
            before.y += s.y;
        }
        all.x += s.x;
        all.y += s.y;
    }
    *total = all;
    return make_int2(v.x + before.x, v.y + before.y);
}

// Volatile reads: counts change by atomics of the same cluster between two barriers.
__device__ __forceinline__ int fresh_load(const int32_t *a) { return *reinterpret_cast<const volatile int32_t *>(a); }

__global__ void __launch_bounds__(kPlanThreads)
kv_resize_plan_kernel(const ResizeParams p)
{
    namespace cg = cooperative_groups;
    extern __shared__ int32_t plan_smem[];
    __shared__ int2 warp_sums[kPlanThreads / 32];
    __shared__ int granted_total;
    int32_t *old_len = plan_smem;                             // [batch]
    int32_t *new_len = old_len + p.batch;                     // [batch], the old length where nothing changes
    int32_t *ask = new_len + p.batch;                         // [batch] inclusive sum of the blocks asked for
    int32_t *copy_at = ask + p.batch;                         // [batch] index of the copy in the list, -1: none, -2: keeps
    cg::cluster_group cluster = cg::this_cluster();
    const int rank = (int)cluster.block_rank(), t = threadIdx.x, T = p.block_tokens;
    const int64_t capacity = (int64_t)p.max_blocks_per_seq * T;
    asm volatile("griddepcontrol.launch_dependents;");
    asm volatile("griddepcontrol.wait;" ::: "memory");

    auto blocks_of = [&](int len) -> int { return (int)(((int64_t)len + T - 1) / T); };
    for (int b = t; b < p.batch; b += kPlanThreads) {
        const int have = p.seq_lens[b], want = p.want_lens[b];
        const bool ok = have >= 0 && have <= capacity && want >= 0 && want <= capacity;
        if (!ok && rank == 0 && p.status) atomicOr(p.status, kFlagSeqLenRange);
        old_len[b] = have;
        new_len[b] = ok ? want : have;
    }
    if (t == 0) granted_total = 0;
    __syncthreads();

    // 1. What shorter lengths no longer need is given back.
    for (int b = rank; b < p.batch; b += kPlanCtas) {
        if (new_len[b] >= old_len[b]) continue;
        const int32_t *row = p.block_table + (int64_t)b * p.max_blocks_per_seq;
        for (int e = blocks_of(new_len[b]) + t; e < blocks_of(old_len[b]); e += kPlanThreads) {
            const int id = row[e];
            if (id < 0 || (int64_t)id >= p.num_phys_blocks) {
                if (p.status) atomicOr(p.status, kFlagBlockRange);
            } else if (atomicSub(p.block_refs + id, 1) <= 0) {
                atomicAdd(p.block_refs + id, 1);              // already free: the counts do not fit the tables
                if (p.status) atomicOr(p.status, kFlagPool);
            }
        }
    }
    cluster.sync();

    // 2. Copy on write.  A growing sequence writes into its last block next; where others list that
    // block too, it takes a copy -- unless all that list it grow, then the last of them keeps it.
    if (rank == 0) {
        bool any = false;
        for (int b = t; b < p.batch; b += kPlanThreads) {
            int spot = -1;
            if (new_len[b] > old_len[b] && old_len[b] % T != 0) {
                const int id = p.block_table[(int64_t)b * p.max_blocks_per_seq + old_len[b] / T];
                if (id < 0 || (int64_t)id >= p.num_phys_blocks) {
                    if (p.status) atomicOr(p.status, kFlagBlockRange);
                } else if (fresh_load(p.block_refs + id) > 1) {
                    spot = id;
                    any = true;
                }
            }
            copy_at[b] = spot;
        }
        if (__syncthreads_or(any)) {
            // every candidate takes its reference back; a count of 0 means that all who list the
            // block are candidates.  The highest of them is elected by a minimum of -1 - b.
            for (int b = t; b < p.batch; b += kPlanThreads)
                if (copy_at[b] >= 0) atomicSub(p.block_refs + copy_at[b], 1);
            __syncthreads();
            for (int b = t; b < p.batch; b += kPlanThreads) ask[b] = copy_at[b] >= 0 && fresh_load(p.block_refs + copy_at[b]) == 0;
            __syncthreads();
            for (int b = t; b < p.batch; b += kPlanThreads)
                if (ask[b]) atomicMin(p.block_refs + copy_at[b], -1 - b);
            __syncthreads();
            for (int b = t; b < p.batch; b += kPlanThreads) ask[b] = ask[b] && fresh_load(p.block_refs + copy_at[b]) == -1 - b;
            __syncthreads();
            for (int b = t; b < p.batch; b += kPlanThreads) {
                if (ask[b]) {                                 // this one keeps the block, as its only owner
                    *reinterpret_cast<volatile int32_t *>(p.block_refs + copy_at[b]) = 1;
                    copy_at[b] = -2;
                }
            }
            __syncthreads();
        }
        for (int b = t; b < p.batch; b += kPlanThreads) {
            const int more = max(0, blocks_of(new_len[b]) - blocks_of(old_len[b]));
            p.counts[b] = copy_at[b] >= 0 ? more + 1 + kCopyBit : copy_at[b] == -2 ? more + kKeepBit : more;
        }
    }
    cluster.sync();

    // 3. Running sums of what is asked for (every block of the cluster has them all), and the free
    // blocks of each block's range of ids.
    int asked = 0, copies = 0;
    for (int b0 = 0; b0 < p.batch; b0 += kPlanThreads) {
        const int b = b0 + t;
        const int c = b < p.batch ? fresh_load(p.counts + b) : 0;
        int2 total;
        const int2 sum = plan_scan(make_int2(c & ~(kCopyBit | kKeepBit), c & kCopyBit ? 1 : 0), warp_sums, &total);
        if (b < p.batch) {
            ask[b] = asked + sum.x;
            copy_at[b] = c & kCopyBit ? copies + sum.y - 1 : c & kKeepBit ? -2 : -1;
        }
        asked += total.x;
        copies += total.y;
    }
    const int64_t slice = ((p.num_phys_blocks + kPlanCtas - 1) / kPlanCtas + 3) / 4 * 4;
    const int64_t from = min((int64_t)rank * slice, p.num_phys_blocks), to = min(from + slice, p.num_phys_blocks);
    int free_here = 0;
    if (asked > 0) {
        int mine = 0;
        for (int64_t i = from + t; i < to; i += kPlanThreads) mine += fresh_load(p.block_refs + i) <= 0;
        int2 total;
        plan_scan(make_int2(mine, 0), warp_sums, &total);
        free_here = total.x;
    }
    if (t == 0) p.slices[rank] = free_here;
    cluster.sync();
    int64_t rank_base = 0, free_total = 0;
    for (int r = 0; r < kPlanCtas; ++r) {
        const int n = fresh_load(p.slices + r);
        if (r < rank) rank_base += n;
        free_total += n;
    }

    // 4. Sequences are served in order until one does not fit; it and all later ones that ask keep
    // what they have.  (The running sums only grow, so one comparison per sequence says it.)  One
    // that keeps a block which earlier sequences leave is refused with them even if it asks for
    // none: it would write where they still read.
    auto blocks_asked = [&](int b) -> int { return b > 0 ? ask[b] - ask[b - 1] : ask[0]; };
    for (int b = t; b < p.batch; b += kPlanThreads)
        if (blocks_asked(b) > 0 && ask[b] <= free_total) atomicMax(&granted_total, ask[b]);
    __syncthreads();
    const int granted = granted_total;

    // 5. The lowest free ids, in order, to the sequences in order.
    int64_t next = rank_base;                                 // rank of this range's next free block
    for (int64_t i0 = from; i0 < to && next < granted; i0 += kPlanThreads) {
        const int64_t id = i0 + t;
        const int is_free = id < to && fresh_load(p.block_refs + id) <= 0;
        int2 total;
        const int2 sum = plan_scan(make_int2(is_free, 0), warp_sums, &total);
        const int64_t place = next + sum.x - 1;
        next += total.x;
        if (is_free && place < granted) {
            int lo = 0, hi = p.batch - 1;                     // the first sequence whose running sum exceeds `place`
            while (lo < hi) {
                const int mid = (lo + hi) / 2;
                if (ask[mid] > place) hi = mid;
                else lo = mid + 1;
            }
            int32_t *row = p.block_table + (int64_t)lo * p.max_blocks_per_seq;
            int nth = (int)(place - (ask[lo] - blocks_asked(lo)));
            p.block_refs[id] = 1;
            if (copy_at[lo] >= 0 && nth == 0) {
                const int e = old_len[lo] / T;
                p.list.pages[2 * copy_at[lo]] = row[e];
                p.list.pages[2 * copy_at[lo] + 1] = (int)id;
                row[e] = (int)id;
            } else {
                row[blocks_of(old_len[lo]) + nth - (copy_at[lo] >= 0 ? 1 : 0)] = (int)id;
            }
        }
    }
    // 6. Lengths; who was not served takes back its reference to the block it would have left.
    if (rank == 0) {
        int served_copies = 0;
        for (int b = t; b < p.batch; b += kPlanThreads) {
            const bool refused = (blocks_asked(b) > 0 || copy_at[b] == -2) && ask[b] > granted;
            p.new_lens[b] = refused ? old_len[b] : new_len[b];
            if (refused && p.status) atomicOr(p.status, kFlagPool);
            if (copy_at[b] >= 0) {
                if (refused) atomicAdd(p.block_refs + p.block_table[(int64_t)b * p.max_blocks_per_seq + old_len[b] / T], 1);
                else served_copies = max(served_copies, copy_at[b] + 1);
            }
        }
        __syncthreads();
        if (t == 0) granted_total = 0;
        __syncthreads();
        atomicMax(&granted_total, served_copies);
        __syncthreads();
        if (t == 0) *p.list.count = granted_total;
    }
}

// ---- deciding a defragmentation --------------------------------------------------------------
struct DefragmentParams {
    const int32_t *block_table;
    int32_t *new_table;           // may be block_table itself
    const int32_t *block_refs;
    int32_t *new_refs;            // may be block_refs itself
    const int32_t *seq_lens;
    int32_t *blocks_used;         // [1]
    int32_t *status;
    int64_t num_phys_blocks;
    int32_t batch, block_tokens, max_blocks_per_seq;
    int32_t *map;                 // [num_phys_blocks] where each block goes
    int32_t *slices;              // [2 * kPlanCtas]
    PageList list;
};

// U blocks are in use.  Those with an id of U or more (in order) go to the free ids below U (in
// order); there are equally many of both.
__global__ void __launch_bounds__(kPlanThreads)
kv_defragment_plan_kernel(const DefragmentParams p)
{
    namespace cg = cooperative_groups;
    __shared__ int2 warp_sums[kPlanThreads / 32];
    cg::cluster_group cluster = cg::this_cluster();
    const int rank = (int)cluster.block_rank(), t = threadIdx.x;
    asm volatile("griddepcontrol.launch_dependents;");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int64_t slice = ((p.num_phys_blocks + kPlanCtas - 1) / kPlanCtas + 3) / 4 * 4;
    const int64_t from = min((int64_t)rank * slice, p.num_phys_blocks), to = min(from + slice, p.num_phys_blocks);

    int mine = 0;
    int2 total;
    for (int64_t i = from + t; i < to; i += kPlanThreads) mine += p.block_refs[i] > 0;
    plan_scan(make_int2(mine, 0), warp_sums, &total);
    if (t == 0) p.slices[rank] = total.x;
    cluster.sync();
    int64_t used = 0, used_before = 0;
    for (int r = 0; r < kPlanCtas; ++r) {
        const int n = fresh_load(p.slices + r);
        if (r < rank) used_before += n;
        used += n;
    }
    // Of the ids before `from`, min(from, U) lie below U; how many of those are free, and how many
    // used ones lie at U or beyond, follows once the range that holds U has counted its two sides.
    int low = 0;
    for (int64_t i = from + t; i < min(to, used); i += kPlanThreads) low += p.block_refs[i] > 0;
    plan_scan(make_int2(low, 0), warp_sums, &total);
    if (t == 0) p.slices[kPlanCtas + rank] = total.x;
    cluster.sync();
    int64_t low_before = 0;                                   // used ids below both U and `from`
    for (int r = 0; r < rank; ++r) low_before += fresh_load(p.slices + kPlanCtas + r);
    int64_t hole = min(from, used) - low_before, mover = used_before - low_before;
    for (int64_t i0 = from; i0 < to; i0 += kPlanThreads) {
        const int64_t id = i0 + t;
        const bool in_use = id < to && p.block_refs[id] > 0;
        const bool is_hole = id < to && id < used && !in_use, moves = in_use && id >= used;
        const int2 sum = plan_scan(make_int2(is_hole, moves), warp_sums, &total);
        if (is_hole) p.list.pages[2 * (hole + sum.x - 1) + 1] = (int)id;
        if (moves) p.list.pages[2 * (mover + sum.y - 1)] = (int)id;
        if (id < to) p.map[id] = in_use && id < used ? (int)id : -1;      // (a hole is no one's, though a mover will lie there)
        hole += total.x;
        mover += total.y;
    }
    if (rank == kPlanCtas - 1 && t == 0) {
        *p.list.count = (int)mover;
        p.slices[0] = (int)mover;
        *p.blocks_used = (int)used;
    }
    cluster.sync();
    const int moved = fresh_load(p.slices);
    for (int i = rank * kPlanThreads + t; i < moved; i += kPlanCtas * kPlanThreads) {
        const int src = fresh_load(p.list.pages + 2 * i), dst = fresh_load(p.list.pages + 2 * i + 1);
        p.map[src] = dst;
        p.new_refs[dst] = p.block_refs[src];                  // dst is free, src is not: no one else reads or writes either
    }
    cluster.sync();                                           // the counts of the moved blocks have been read
    for (int64_t i = from + t; i < to; i += kPlanThreads) {
        if (i >= used) p.new_refs[i] = 0;
        else if (p.block_refs != p.new_refs && p.block_refs[i] > 0) p.new_refs[i] = p.block_refs[i];
    }
}

// ---- moving pages ----------------------------------------------------------------------------
constexpr int kMoveThreads = 256;
constexpr int kMoveUnroll = 4;
constexpr int kMoveSegs = kMoveThreads * kMoveUnroll;         // 16 KiB of one page per block and step

// Pages of all layers, K and V, from the list: the work is cut into 16 KiB pieces that the blocks
// of one grid take in turn; each thread has four 16-byte loads in flight before its stores.
// kRemap: the blocks first rewrite the tables (the defragmentation's second half).
template <bool kRemap>
__global__ void __launch_bounds__(kMoveThreads)
kv_move_pages_kernel(const PageList list, int layers, int64_t page_segs, int64_t num_phys_blocks, int32_t *status,
                     const DefragmentParams d, const __grid_constant__ LayerCaches caches)
{
    asm volatile("griddepcontrol.launch_dependents;");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    if (kRemap) {
        const int64_t entries = (int64_t)d.batch * d.max_blocks_per_seq;
        for (int64_t i = (int64_t)blockIdx.x * kMoveThreads + threadIdx.x; i < entries; i += (int64_t)gridDim.x * kMoveThreads) {
            const int b = (int)(i / d.max_blocks_per_seq), e = (int)(i - (int64_t)b * d.max_blocks_per_seq);
            const int len = d.seq_lens[b];
            int id = d.block_table[i];
            if (len < 0 || (int64_t)len > (int64_t)d.max_blocks_per_seq * d.block_tokens) {
                if (e == 0 && status) atomicOr(status, kFlagSeqLenRange);
            } else if ((int64_t)e * d.block_tokens < len) {
                if (id < 0 || (int64_t)id >= num_phys_blocks) {
                    if (status) atomicOr(status, kFlagBlockRange);
                } else {
                    const int to = d.map[id];
                    if (to < 0 && status) atomicOr(status, kFlagPool);      // a listed block that counts as free
                    if (to >= 0) id = to;
                }
            }
            d.new_table[i] = id;
        }
    }
    const int n = *list.count;
    const int64_t pieces = (page_segs + kMoveSegs - 1) / kMoveSegs;
    const int64_t work = (int64_t)n * layers * 2 * pieces;
    for (int64_t w = blockIdx.x; w < work; w += gridDim.x) {
        const int64_t page = w / pieces;
        const int64_t seg0 = (w - page * pieces) * kMoveSegs + threadIdx.x;
        const int i = (int)(page / (2 * layers)), which = (int)(page - (int64_t)i * 2 * layers);
        const int src = list.pages[2 * i], dst = list.pages[2 * i + 1];
        if (!bounds_ok(src >= 0 && src < num_phys_blocks && dst >= 0 && dst < num_phys_blocks, status)) continue;
        uint4 *cache = (which & 1) ? caches.v[which >> 1] : caches.k[which >> 1];
        const uint4 *from = cache + (int64_t)src * page_segs;
        uint4 *to = cache + (int64_t)dst * page_segs;
        uint4 x[kMoveUnroll];
#pragma unroll
        for (int u = 0; u < kMoveUnroll; ++u)
            if (seg0 + u * kMoveThreads < page_segs) x[u] = from[seg0 + u * kMoveThreads];
#pragma unroll
        for (int u = 0; u < kMoveUnroll; ++u)
            if (seg0 + u * kMoveThreads < page_segs) to[seg0 + u * kMoveThreads] = x[u];
    }
}

}  // namespace instinfer
