// Draft trees for sm_100a: the ancestors' bit masks that tree attention reads, and the
// verification of a tree of drafted tokens against the target's probabilities.
//
// Verification is recursive rejection sampling.  At node v, w = p_v (the target's distribution
// after v) and Z = 1; the children c of v are tried in index order: c is taken if
//     u_c q_v(x_c) Z < w(x_c),
// and the walk goes on from c; otherwise w <- max(w - Z q_v, 0), Z <- sum w, which is Z times the
// residual distribution (an empty residual, sum 0, leaves w and Z as they were).  Where no child
// is taken, the next token is the first i with w_0 + ... + w_i > u_0 sum w.  If the children of v
// were drawn from q_v independently, the emitted tokens are distributed as the target's.  Without
// draft distributions q_v is one-hot at x_c (drafts that were not sampled).
//
// Everything is decided in 64 bits: a decision compares numbers that differ by as little as one
// rounding, and the sums run over a vocabulary.  Only the node where the walk ends (and nodes with
// a rejected child before a later one) needs passes over whole rows, so the work is a row or two
// of p and q per sequence: latency for one sequence, HBM bandwidth for many.  A cluster of up to
// 8 blocks shares a sequence's rows and holds the current node's in its registers; all blocks walk the
// tree alike on the few gathered values, and exchange only their partial sums, through distributed
// shared memory.
//
// Measured: one sequence (8 nodes, 32,000 fp32 probabilities a row) 8.2 us a call and of the GPU's time in a
// graph: a chain of loads, passes and exchanges; 64 sequences (32 nodes, 50,257 bf16) 36 to 39 us, bound by the passes of
// the 1.7 waves of clusters: an exchange of sums among 8 blocks is some 1.5 us, a residual pass in 64 bits as much
// again.  Rows that are streamed: 16 sequences (8 nodes) of 151,936 bf16 76 us and of 256,000 118 us, where 131,064
// held ones take 23 us; one sequence of 256,000 fp32 30 us.
#pragma once

#include <cooperative_groups.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "kv_pages_kernels.cuh"

namespace instinfer {

// ---- ancestors -------------------------------------------------------------------------------
// One block per sequence, one thread per node: its bits are itself and every node on its way to a
// root.  Parents come before their children, so a walk takes at most its node's index in steps.
__global__ void __launch_bounds__(kMaxTreeTokens)
tree_mask_kernel(uint64_t *mask, const int32_t *parents, const int32_t *tree_lens, int32_t tree_tokens, int32_t words,
                 int32_t *status)
{
    __shared__ int up[kMaxTreeTokens];
    const int b = blockIdx.x, t = threadIdx.x;
    asm volatile("griddepcontrol.launch_dependents;");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    int nodes = tree_lens ? tree_lens[b] : tree_tokens;
    bool bad = nodes < 0 || nodes > tree_tokens;
    if (bad) nodes = 0;
    if (t < nodes) {
        int parent = parents[(int64_t)b * tree_tokens + t];
        if (parent < -1 || parent >= t) {                     // treated as a root
            parent = -1;
            bad = true;
        }
        up[t] = parent;
    }
    if (bad && status) atomicOr(status, kFlagTreeRange);
    __syncthreads();
    uint64_t bits[2] = {0, 0};
    if (t < nodes)
        for (int a = t; a >= 0; a = up[a]) bits[a >> 6] |= (uint64_t)1 << (a & 63);
    if (t < tree_tokens)
        for (int w = 0; w < words; ++w) mask[((int64_t)b * tree_tokens + t) * words + w] = bits[w];
}

// ---- verification ----------------------------------------------------------------------------
struct VerifyParams {
    int32_t *path;                // [batch, tree_tokens]
    int32_t *path_lens;           // [batch]
    int32_t *out_tokens;          // [batch, tree_tokens]
    const void *target;           // rows of `vocab` probabilities, row_stride elements apart
    const void *draft;            // the same rows of the draft's distributions, nullable
    const int32_t *tokens;        // [batch, tree_tokens]
    const int32_t *parents;
    const int32_t *tree_lens;     // nullable
    const float *uniforms;        // [batch, tree_tokens]
    int32_t *status;
    int64_t row_stride;
    int32_t tree_tokens, vocab;
};

constexpr int kVerifyThreads = 256;
constexpr int kVerifyWarps = kVerifyThreads / 32;
constexpr int kVerifyMaxCtas = 8;

// A probability as the verification sees it: what is not a positive finite number counts as 0.
__device__ __forceinline__ double clean(float x) { return x > 0.f && x < INFINITY ? (double)x : 0.0; }
__device__ __forceinline__ float widen(float x) { return x; }
__device__ __forceinline__ float widen(__half x) { return __half2float(x); }
__device__ __forceinline__ float widen(__nv_bfloat16 x) { return __bfloat162float(x); }

// 16 bytes of a row: group g holds elements g * kVec - shift ..., where `shift` makes groups fall
// on 16-byte boundaries of memory (rows of an odd vocabulary start anywhere); elements outside
// the row read as 0.
template <typename E>
struct RowReader {
    static constexpr int kVec = 16 / (int)sizeof(E);
    const E *row;
    int vocab, shift;
    __device__ __forceinline__ RowReader(const void *base, int64_t offset, int vocab_)
        : row(static_cast<const E *>(base) + offset), vocab(vocab_),
          shift((int)((reinterpret_cast<uintptr_t>(row) & 15u) / sizeof(E))) {}
    __device__ __forceinline__ int groups() const { return (vocab + shift + kVec - 1) / kVec; }
    __device__ __forceinline__ uint4 raw(int g) const
    {
        const int first = g * kVec - shift;
        if (first >= 0 && first + kVec <= vocab) return *reinterpret_cast<const uint4 *>(row + first);
        uint4 some = make_uint4(0u, 0u, 0u, 0u);
        E *e = reinterpret_cast<E *>(&some);
#pragma unroll
        for (int i = 0; i < kVec; ++i)
            if (first + i >= 0 && first + i < vocab) e[i] = row[first + i];
        return some;
    }
    static __device__ __forceinline__ double value(const uint4 &group, int i) { return clean(widen(reinterpret_cast<const E *>(&group)[i])); }
    __device__ __forceinline__ void load(int g, float (&x)[kVec]) const
    {
        const uint4 group = raw(g);
#pragma unroll
        for (int i = 0; i < kVec; ++i) x[i] = widen(reinterpret_cast<const E *>(&group)[i]);
    }
};

__device__ __forceinline__ double warp_sum(double v)
{
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}

// The weights w of the walk's current node in the registers of the cluster: a warp (one of `pieces`, in the order of
// the row) holds a run of 16-byte groups, thread `lane` the groups lane, lane + 32, ... of it.  A residual then
// costs three 64-bit operations per element and no memory, whatever the number of earlier ones.
template <typename E, int kPer>
struct HeldWeights {
    static constexpr int kVec = RowReader<E>::kVec;
    double w[kPer * kVec];
    uint4 q[kPer];                 // as they lie in memory: registers decide how many sequences run at once
    int first;                     // group of this thread's w[0 .. kVec)
    int shift;

    __device__ __forceinline__ int element(int i, int e) const { return (first + 32 * i) * kVec - shift + e; }
    __device__ __forceinline__ void load(const VerifyParams &p, int64_t offset, int piece, int pieces, int lane, bool with_q)
    {
        const RowReader<E> pr(p.target, offset, p.vocab), qr(with_q ? p.draft : p.target, offset, p.vocab);
        const int groups = pr.groups();
        const int g0 = (int)((int64_t)groups * piece / pieces), g1 = (int)((int64_t)groups * (piece + 1) / pieces);
        first = g0 + lane;
        shift = pr.shift;
        uint4 x[kPer];
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            x[i] = q[i] = make_uint4(0u, 0u, 0u, 0u);
            if (first + 32 * i < g1) {
                x[i] = pr.raw(first + 32 * i);
                if (with_q) q[i] = qr.raw(first + 32 * i);
            }
        }
#pragma unroll
        for (int i = 0; i < kPer * kVec; ++i) w[i] = RowReader<E>::value(x[i / kVec], i % kVec);
    }
    // w <- max(w - total q, 0); a draft that was not sampled has q one-hot at `token`
    __device__ __forceinline__ void reduce(double total, bool sampled, int token)
    {
        if (sampled) {
#pragma unroll
            for (int i = 0; i < kPer * kVec; ++i) w[i] = fmax(__dsub_rn(w[i], __dmul_rn(total, RowReader<E>::value(q[i / kVec], i % kVec))), 0.0);
        } else {
#pragma unroll
            for (int i = 0; i < kPer * kVec; ++i)
                if (element(i / kVec, i % kVec) == token) w[i] = fmax(__dsub_rn(w[i], total), 0.0);
        }
    }
    __device__ __forceinline__ double sum() const
    {
        double s[4] = {0.0, 0.0, 0.0, 0.0};
#pragma unroll
        for (int i = 0; i < kPer * kVec; ++i) s[i & 3] += w[i];
        return (s[0] + s[1]) + (s[2] + s[3]);
    }
};

// kPer: 16-byte groups of a row that a thread holds.
template <typename E, int kPer, int kThreadsOf>
__global__ void __launch_bounds__(kThreadsOf, 512 / kThreadsOf)
verify_tree_kernel(const VerifyParams p)
{
    namespace cg = cooperative_groups;
    constexpr int kVec = RowReader<E>::kVec, kWarpsOf = kThreadsOf / 32, kMaxPieces = kVerifyMaxCtas * kWarpsOf;
    cg::cluster_group cluster = cg::this_cluster();
    __shared__ int s_parent[kMaxTreeTokens], s_token[kMaxTreeTokens], s_path[kMaxTreeTokens], s_rejected[kMaxTreeTokens];
    __shared__ double s_target[kMaxTreeTokens], s_draft[kMaxTreeTokens], s_u[kMaxTreeTokens], s_total[kMaxTreeTokens];
    __shared__ double s_sums[2][kMaxPieces];                            // every warp's share of a pass, by the pass's parity
    const int ctas = (int)cluster.num_blocks(), rank = (int)cluster.block_rank();
    const int b = blockIdx.x / ctas, t = threadIdx.x, lane = t & 31, warp = t >> 5;
    const int N = p.tree_tokens;
    asm volatile("griddepcontrol.launch_dependents;");
    asm volatile("griddepcontrol.wait;" ::: "memory");

    const int64_t first_row = (int64_t)b * N;
    int nodes = p.tree_lens ? p.tree_lens[b] : N;
    if (nodes < 0 || nodes > N) {
        if (rank == 0 && t == 0 && p.status) atomicOr(p.status, kFlagTreeRange);
        nodes = 0;
    }
    // The values that the walk compares: each node's token under its parent's two distributions.
    if (t < N) {
        int parent = -1, token = -1;
        double pt = 0.0, qt = 1.0;
        if (t < nodes) {
            token = p.tokens[first_row + t];
            parent = p.parents[first_row + t];
            s_u[t] = (double)p.uniforms[first_row + t];
            const bool token_ok = token >= 0 && token < p.vocab;
            if (t > 0) {                                      // the root is given, not tried
                if (parent < 0 || parent >= t || !token_ok) {
                    if (rank == 0 && p.status) atomicOr(p.status, kFlagTreeRange);
                    parent = -1;                              // never tried
                } else {
                    const int64_t at = (first_row + parent) * p.row_stride + token;
                    const E x = static_cast<const E *>(p.target)[at];
                    if (p.draft) qt = clean(widen(static_cast<const E *>(p.draft)[at]));
                    pt = clean(widen(x));
                }
            }
        }
        s_parent[t] = t > 0 ? parent : -1;
        s_token[t] = token;
        s_target[t] = pt;
        s_draft[t] = qt;
    }
    cluster.sync();                                           // also: every block runs before its shared memory is written to

    int at = 0, kept = nodes > 0 ? 1 : 0, pass = 0;
    if (nodes > 0) {
        // ---- the walk: the same in every thread of the cluster ----
        const int pieces = ctas * kWarpsOf, piece = rank * kWarpsOf + warp;
        HeldWeights<E, kPer> held;
        int rejected = 0;                                     // residuals taken at the current node, from s_total[0 .. rejected)
        bool loaded = false, summed = false;                  // the current w is held; its sums are in s_sums
        double total = 1.0;
        auto load = [&]() {
            held.load(p, (first_row + at) * p.row_stride, piece, pieces, lane, p.draft != nullptr);
            for (int k = 0; k < rejected; ++k) held.reduce(s_total[k], p.draft != nullptr, s_rejected[k]);
            loaded = true;
        };
        // The sum of w over the vocabulary; the warps' shares stay in s_sums.
        auto sum_row = [&]() -> double {
            const double sum = warp_sum(held.sum());
            const int parity = pass & 1;
            if (lane < ctas) cluster.map_shared_rank(&s_sums[0][0], lane)[parity * kMaxPieces + piece] = sum;
            cluster.sync();
            ++pass;
            double mine = 0.0;
            for (int i = lane; i < pieces; i += 32) mine += s_sums[parity][i];
            return warp_sum(mine);
        };
        if (t == 0) s_path[0] = 0;
        for (int c = 1; c < nodes;) {
            // the next child of `at` from c on
            int next = nodes;
            for (int base = c & ~31; base < nodes && next == nodes; base += 32) {
                const int n = base + lane;
                const unsigned hit = __ballot_sync(0xffffffffu, n >= c && n < nodes && s_parent[n] == at);
                if (hit) next = base + __ffs(hit) - 1;
            }
            if (next == nodes) break;
            // w at the child's token: its value after the residuals so far
            const double q = s_draft[next];
            double w = s_target[next];
            for (int k = 0; k < rejected; ++k) {
                const double qk = p.draft ? q : (s_token[next] == s_rejected[k] ? 1.0 : 0.0);
                w = fmax(__dsub_rn(w, __dmul_rn(s_total[k], qk)), 0.0);
            }
            if (s_u[next] * q * total < w) {
                at = next;
                if (t == 0) s_path[kept] = next;
                ++kept;
                rejected = 0;
                total = 1.0;
                loaded = summed = false;
            } else {
                if (!loaded) load();
                __syncthreads();                              // earlier readers of the lists are done
                if (t == 0) {
                    s_total[rejected] = total;
                    s_rejected[rejected] = s_token[next];
                }
                __syncthreads();
                held.reduce(total, p.draft != nullptr, s_token[next]);
                const double left = sum_row();
                summed = left > 0.0;
                if (summed) {
                    total = left;
                    ++rejected;
                } else {
                    loaded = false;                           // an empty residual: w stays as it was
                }
            }
            c = next + 1;
        }
        if (!loaded) load();
        if (!summed) total = sum_row();
        // ---- the next token: the first element at which the running sum exceeds u_0 * total ----
        const double *sums = s_sums[(pass - 1) & 1];
        const double goal = s_u[0] * total;
        double before = 0.0, before_last = 0.0;
        int chosen = -1, last_live = -1;
        for (int i0 = 0; i0 < pieces && chosen < 0; i0 += 32) {       // 32 shares at a time
            const double mine = i0 + lane < pieces ? sums[i0 + lane] : 0.0;
            double run = mine;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const double up = __shfl_up_sync(0xffffffffu, run, o);
                if (lane >= o) run += up;
            }
            const unsigned live = __ballot_sync(0xffffffffu, mine > 0.0);
            const unsigned over = __ballot_sync(0xffffffffu, mine > 0.0 && before + run > goal);
            const int pick = over ? __ffs(over) - 1 : live ? 31 - __clz(live) : 0;
            const double prior = before + __shfl_sync(0xffffffffu, run - mine, pick);
            if (over) {
                chosen = i0 + pick;
                before = prior;
            } else {
                if (live) {
                    last_live = i0 + pick;
                    before_last = prior;
                }
                before += __shfl_sync(0xffffffffu, run, 31);
            }
        }
        if (chosen < 0) {                                     // u_0 is not below 1
            chosen = last_live;
            before = before_last;
        }
        if (chosen < 0) {                                     // no positive probability at all
            if (rank == 0 && t == 0) {
                p.out_tokens[first_row + kept - 1] = -1;
                if (p.status) atomicOr(p.status, kFlagTreeRange);
            }
        } else if (chosen == piece) {
            int found = -1, last = -1;                        // `last`: the last element with any weight
#pragma unroll
            for (int i = 0; i < kPer; ++i) {
                if (found >= 0) continue;
                double mine = 0.0;
                int mine_last = -1;
#pragma unroll
                for (int e = 0; e < kVec; ++e) {
                    mine += held.w[i * kVec + e];
                    if (held.w[i * kVec + e] > 0.0) mine_last = held.element(i, e);
                }
                double run = mine;                            // inclusive over the lanes
#pragma unroll
                for (int o = 1; o < 32; o <<= 1) {
                    const double up = __shfl_up_sync(0xffffffffu, run, o);
                    if (lane >= o) run += up;
                }
                double upto = before + (run - mine);
                int here = -1;
#pragma unroll
                for (int e = 0; e < kVec; ++e) {
                    upto += held.w[i * kVec + e];
                    if (here < 0 && held.w[i * kVec + e] > 0.0 && upto > goal) here = held.element(i, e);
                }
                const unsigned hit = __ballot_sync(0xffffffffu, here >= 0);
                if (hit) found = __shfl_sync(0xffffffffu, here, __ffs(hit) - 1);
                last = max(last, __reduce_max_sync(0xffffffffu, mine_last));
                before += __shfl_sync(0xffffffffu, run, 31);
            }
            if (lane == 0) p.out_tokens[first_row + kept - 1] = found >= 0 ? found : last;
        }
    }
    __syncthreads();
    if (rank == 0) {
        if (t < N) {
            p.path[first_row + t] = t < kept ? s_path[t] : -1;
            if (t < kept - 1) p.out_tokens[first_row + t] = s_token[s_path[t + 1]];
            else if (t >= kept) p.out_tokens[first_row + t] = -1;
        }
        if (t == 0) p.path_lens[b] = kept;
    }
}

// The same with the rows read again for every residual: vocabularies that the registers of a cluster do not hold.
template <typename E>
__global__ void __launch_bounds__(kVerifyThreads)
verify_tree_streamed_kernel(const VerifyParams p)
{
    namespace cg = cooperative_groups;
    constexpr int kVec = RowReader<E>::kVec;
    cg::cluster_group cluster = cg::this_cluster();
    __shared__ int s_parent[kMaxTreeTokens], s_token[kMaxTreeTokens], s_path[kMaxTreeTokens], s_rejected[kMaxTreeTokens];
    __shared__ double s_target[kMaxTreeTokens], s_draft[kMaxTreeTokens], s_u[kMaxTreeTokens], s_total[kMaxTreeTokens];
    __shared__ double s_sums[2][kVerifyMaxCtas * kVerifyWarps];         // every warp's share of a pass, by the pass's parity
    const int ctas = (int)cluster.num_blocks(), rank = (int)cluster.block_rank();
    const int b = blockIdx.x / ctas, t = threadIdx.x, lane = t & 31, warp = t >> 5;
    const int N = p.tree_tokens;
    asm volatile("griddepcontrol.launch_dependents;");
    asm volatile("griddepcontrol.wait;" ::: "memory");

    const int64_t first_row = (int64_t)b * N;
    int nodes = p.tree_lens ? p.tree_lens[b] : N;
    if (nodes < 0 || nodes > N) {
        if (rank == 0 && t == 0 && p.status) atomicOr(p.status, kFlagTreeRange);
        nodes = 0;
    }
    // The values that the walk compares: each node's token under its parent's two distributions.
    if (t < N) {
        int parent = -1, token = -1;
        double pt = 0.0, qt = 1.0;
        if (t < nodes) {
            token = p.tokens[first_row + t];
            parent = p.parents[first_row + t];
            const bool token_ok = token >= 0 && token < p.vocab;
            if (t > 0) {                                      // the root is given, not tried
                if (parent < 0 || parent >= t || !token_ok) {
                    if (rank == 0 && p.status) atomicOr(p.status, kFlagTreeRange);
                    parent = -1;                              // never tried
                } else {
                    const int64_t at = (first_row + parent) * p.row_stride + token;
                    pt = clean(widen(static_cast<const E *>(p.target)[at]));
                    if (p.draft) qt = clean(widen(static_cast<const E *>(p.draft)[at]));
                }
            }
            s_u[t] = (double)p.uniforms[first_row + t];
        }
        s_parent[t] = t > 0 ? parent : -1;
        s_token[t] = token;
        s_target[t] = pt;
        s_draft[t] = qt;
    }
    cluster.sync();                                           // also: every block runs before its shared memory is written to

    int at = 0, kept = nodes > 0 ? 1 : 0, pass = 0;
    if (nodes > 0) {
        // ---- the walk: the same in every thread of the cluster ----
        int rejected = 0;                                     // residuals taken at the current node: s_total[0 .. rejected)
        bool summed = false;                                  // the sums of the current w are in s_sums
        double total = 1.0;
        // w at one element of the current node, from its p and q values
        auto residual = [&](double w, double q, int element) -> double {
            for (int k = 0; k < rejected; ++k) {
                const double qk = p.draft ? q : (element == s_rejected[k] ? 1.0 : 0.0);
                w = fmax(__dsub_rn(w, __dmul_rn(s_total[k], qk)), 0.0);
            }
            return w;
        };
        // Sums of w over the vocabulary: a warp's share of the row is a run of groups, so that the
        // sums of the warps in order are those of consecutive pieces of the row.
        const int pieces = ctas * kVerifyWarps, piece = rank * kVerifyWarps + warp;
        auto sum_row = [&]() -> double {
            const int64_t offset = (first_row + at) * p.row_stride;
            const RowReader<E> pr(p.target, offset, p.vocab), qr(p.draft ? p.draft : p.target, offset, p.vocab);
            const int groups = pr.groups();
            const int g0 = (int)((int64_t)groups * piece / pieces), g1 = (int)((int64_t)groups * (piece + 1) / pieces);
            const bool read_q = p.draft != nullptr && rejected > 0;
            double sum = 0.0;
            for (int g = g0 + lane; g < g1; g += 32) {
                float x[kVec], y[kVec];
                pr.load(g, x);
                if (read_q) qr.load(g, y);
#pragma unroll
                for (int i = 0; i < kVec; ++i)
                    sum += residual(clean(x[i]), read_q ? clean(y[i]) : 0.0, g * kVec - pr.shift + i);
            }
            sum = warp_sum(sum);
            const int parity = pass & 1;
            if (lane < ctas) cluster.map_shared_rank(&s_sums[0][0], lane)[parity * kVerifyMaxCtas * kVerifyWarps + piece] = sum;
            cluster.sync();
            ++pass;
            const double *sums = s_sums[parity];
            return warp_sum((lane < pieces ? sums[lane] : 0.0) + (lane + 32 < pieces ? sums[lane + 32] : 0.0));
        };
        if (t == 0) s_path[0] = 0;
        for (int c = 1; c < nodes;) {
            // the next child of `at` from c on
            int next = nodes;
            for (int base = c & ~31; base < nodes && next == nodes; base += 32) {
                const int n = base + lane;
                const unsigned hit = __ballot_sync(0xffffffffu, n >= c && n < nodes && s_parent[n] == at);
                if (hit) next = base + __ffs(hit) - 1;
            }
            if (next == nodes) break;
            const double q = s_draft[next];
            const double w = residual(s_target[next], q, s_token[next]);
            if (s_u[next] * q * total < w) {
                at = next;
                if (t == 0) s_path[kept] = next;
                ++kept;
                rejected = 0;
                total = 1.0;
                summed = false;
            } else {
                __syncthreads();                              // earlier readers of the lists are done
                if (t == 0) {
                    s_total[rejected] = total;
                    s_rejected[rejected] = s_token[next];
                }
                __syncthreads();
                ++rejected;
                const double left = sum_row();
                summed = left > 0.0;
                if (summed) total = left;
                else --rejected;                              // an empty residual: w stays as it was
            }
            c = next + 1;
        }
        if (!summed) total = sum_row();
        // ---- the next token: the first element at which the running sum exceeds u_0 * total ----
        const double *sums = s_sums[(pass - 1) & 1];
        const double goal = s_u[0] * total;
        double before = 0.0;
        int chosen = -1, last_live = -1;
        double before_last = 0.0;
        for (int i = 0; i < pieces; ++i) {
            const double s = sums[i];
            if (s > 0.0) {
                last_live = i;
                before_last = before;
                if (chosen < 0 && before + s > goal) {
                    chosen = i;
                    break;
                }
            }
            before += s;
        }
        if (chosen < 0) {                                     // u_0 is not below 1
            chosen = last_live;
            before = before_last;
        }
        if (chosen < 0) {                                     // no positive probability at all
            if (rank == 0 && t == 0) {
                p.out_tokens[first_row + kept - 1] = -1;
                if (p.status) atomicOr(p.status, kFlagTreeRange);
            }
        } else if (chosen == piece) {
            const int64_t offset = (first_row + at) * p.row_stride;
            const RowReader<E> pr(p.target, offset, p.vocab), qr(p.draft ? p.draft : p.target, offset, p.vocab);
            const int groups = pr.groups();
            const int g0 = (int)((int64_t)groups * piece / pieces), g1 = (int)((int64_t)groups * (piece + 1) / pieces);
            const bool read_q = p.draft != nullptr && rejected > 0;
            int found = -1, last = -1;                        // `last`: the last element with any weight
            for (int g = g0; g < g1 && found < 0; g += 32) {
                double w[kVec], mine = 0.0;
                float x[kVec], y[kVec];
                const bool live = g + lane < g1;
                if (live) pr.load(g + lane, x);
                if (live && read_q) qr.load(g + lane, y);
                int mine_last = -1;
#pragma unroll
                for (int i = 0; i < kVec; ++i) {
                    const int element = (g + lane) * kVec - pr.shift + i;
                    w[i] = live ? residual(clean(x[i]), read_q ? clean(y[i]) : 0.0, element) : 0.0;
                    if (w[i] > 0.0) mine_last = element;
                    mine += w[i];
                }
                double run = mine;                            // inclusive over the lanes
#pragma unroll
                for (int o = 1; o < 32; o <<= 1) {
                    const double up = __shfl_up_sync(0xffffffffu, run, o);
                    if (lane >= o) run += up;
                }
                double upto = before + (run - mine);
                int here = -1;
#pragma unroll
                for (int i = 0; i < kVec; ++i) {
                    upto += w[i];
                    if (here < 0 && w[i] > 0.0 && upto > goal) here = (g + lane) * kVec - pr.shift + i;
                }
                const unsigned hit = __ballot_sync(0xffffffffu, here >= 0);
                if (hit) found = __shfl_sync(0xffffffffu, here, __ffs(hit) - 1);
                last = max(last, (int)__reduce_max_sync(0xffffffffu, mine_last));
                before += __shfl_sync(0xffffffffu, run, 31);
            }
            if (lane == 0) p.out_tokens[first_row + kept - 1] = found >= 0 ? found : last;
        }
    }
    __syncthreads();
    if (rank == 0) {
        if (t < N) {
            p.path[first_row + t] = t < kept ? s_path[t] : -1;
            if (t < kept - 1) p.out_tokens[first_row + t] = s_token[s_path[t + 1]];
            else if (t >= kept) p.out_tokens[first_row + t] = -1;
        }
        if (t == 0) p.path_lens[b] = kept;
    }
}

}  // namespace instinfer
