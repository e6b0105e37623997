// From a step's logits to the probabilities that verification and sampling take, for sm_100a.
//
// For row t of sequence b and token i, with n_i how often i was said (the output part of the history, and the drafted
// tokens that node t sees) and s_i whether it was said or prompted:
//   z = logit;  s_i: z > 0 ? z / r : z r;  z -= n_i f + [n_i > 0] p;  z += the sequence's biases of i;  not allowed: -inf
//   probability_i = exp((z_i - max z) / T) / sum_j exp((z_j - max z) / T),   T = 0: 1 at the lowest i of the largest z
// in 32 bits, rounded once.
//
// Bound by bytes (a row is read once and written once) and, for few rows, by the chain of steps.  A cluster of 1, 2, 4
// or 8 blocks has a row; a thread keeps its logits in registers from the first read to the last write, so nothing is
// read twice.  Counts need random access: a table of 32-bit words in shared memory, one per token of the block's slice,
// that the history is scattered into (low bits: times said, two flag bits: prompted, biased) while the logits are on
// their way.  Biases are so few that a flagged token looks its own up in the list, in the list's order, which makes
// tokens that are listed twice deterministic.  The blocks exchange a maximum, a sum of exponentials against their own
// maximum and the place of the maximum, once.
#pragma once

#include <cooperative_groups.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "tree_common.cuh"

namespace instinfer {

constexpr int kFlagTokenRange = 64;
constexpr int kLogitThreads = 512;
constexpr int kLogitWarps = kLogitThreads / 32;
constexpr int kLogitMaxCtas = 8;
constexpr int kLogitMaxBias = 256;        // INSTINFER_MAX_BIAS
constexpr unsigned kLogitPrompted = 1u << 31, kLogitBiased = 1u << 30;

struct LogitParams {
    void *out;
    const void *logits;
    const int32_t *tokens;         // nullable [batch, max_tokens]
    const int32_t *token_lens;     // nullable: max_tokens each
    const int32_t *prompt_lens;    // nullable: 0 each
    const float *penalties;        // nullable [batch, 3]: repetition, frequency, presence
    const int32_t *draft_tokens;   // nullable [batch, tree_tokens]
    const uint64_t *tree_mask;     // nullable: a chain
    const int32_t *tree_lens;      // nullable
    const int32_t *bias_tokens;    // nullable [batch, max_bias]
    const float *bias_values;
    const uint32_t *allowed;       // nullable [batch, tree_tokens, words]
    const float *temperatures;     // nullable [batch]: 1
    int32_t *status;
    int64_t row_stride, out_stride;
    int32_t out_type;              // 0 fp32, 1 fp16, 2 bf16
    int32_t max_tokens, max_bias;
    int32_t tree_tokens, vocab;
    int32_t slice;                 // tokens of a block
    int32_t probabilities;         // 0: z / T itself
};

template <typename E>
__device__ __forceinline__ float logit_value(E x)
{
    if constexpr (sizeof(E) == 4) return x;
    else if constexpr (__is_same(E, __half)) return __half2float(x);
    else return __bfloat162float(x);
}
// kVec (1 or 4) values from a kVec-aligned place.
template <typename E, int kVec>
__device__ __forceinline__ void logit_load(const E *from, float (&x)[kVec])
{
    if constexpr (kVec == 1) {
        x[0] = logit_value(*from);
    } else if constexpr (sizeof(E) == 4) {
        *reinterpret_cast<float4 *>(x) = *reinterpret_cast<const float4 *>(from);
    } else {
        const uint2 raw = *reinterpret_cast<const uint2 *>(from);
        const E *four = reinterpret_cast<const E *>(&raw);
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = logit_value(four[i]);
    }
}
template <typename E>
__device__ __forceinline__ unsigned logit_pack(float a, float b)
{
    if constexpr (__is_same(E, __half)) {
        const __half2 two = __floats2half2_rn(a, b);
        return *reinterpret_cast<const unsigned *>(&two);
    } else {
        const __nv_bfloat162 two = __floats2bfloat162_rn(a, b);
        return *reinterpret_cast<const unsigned *>(&two);
    }
}
template <int kVec>
__device__ __forceinline__ void logit_store(void *out, int type, int64_t at, const float (&x)[kVec], int n)
{
    if (kVec == 4 && n == 4) {
        if (type == 0) *reinterpret_cast<float4 *>(static_cast<float *>(out) + at) = *reinterpret_cast<const float4 *>(x);
        else if (type == 1) *reinterpret_cast<uint2 *>(static_cast<__half *>(out) + at) = make_uint2(logit_pack<__half>(x[0], x[1]), logit_pack<__half>(x[kVec / 2], x[kVec - 1]));
        else *reinterpret_cast<uint2 *>(static_cast<__nv_bfloat16 *>(out) + at) = make_uint2(logit_pack<__nv_bfloat16>(x[0], x[1]), logit_pack<__nv_bfloat16>(x[kVec / 2], x[kVec - 1]));
        return;
    }
#pragma unroll
    for (int i = 0; i < kVec; ++i) {
        if (i >= n) break;
        if (type == 0) static_cast<float *>(out)[at + i] = x[i];
        else if (type == 1) static_cast<__half *>(out)[at + i] = __float2half_rn(x[i]);
        else static_cast<__nv_bfloat16 *>(out)[at + i] = __float2bfloat16_rn(x[i]);
    }
}

struct LogitBest {
    float value;
    int at;
    __device__ __forceinline__ void take(float v, int i)
    {
        if (v > value || (v == value && i < at)) {
            value = v;
            at = i;
        }
    }
};

// kHeld: logits of a thread; kVec: how many of them lie together (4 where every row starts on a 4-element boundary).
template <typename E, int kHeld, int kVec>
__global__ void __launch_bounds__(kLogitThreads, kHeld <= 32 ? 2 : 1)
process_logits_kernel(const LogitParams p)
{
    namespace cg = cooperative_groups;
    constexpr int kGroups = kHeld / kVec;
    extern __shared__ unsigned table[];                       // [slice], where there is anything to look up
    __shared__ LogitBest best_by_warp[kLogitWarps], best_by_cta[kLogitMaxCtas];
    __shared__ float sum_by_warp[kLogitWarps], sum_by_cta[kLogitMaxCtas];
    __shared__ int bias_tokens[kLogitMaxBias];
    __shared__ float bias_values[kLogitMaxBias];
    const cg::cluster_group cluster = cg::this_cluster();
    const int ctas = (int)cluster.num_blocks(), rank = (int)cluster.block_rank();
    const int64_t row = blockIdx.x / ctas;
    const int b = (int)(row / p.tree_tokens), t = (int)(row - (int64_t)b * p.tree_tokens);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");     // (waited for before the blocks write to one another)
    asm volatile("griddepcontrol.launch_dependents;");
    asm volatile("griddepcontrol.wait;" ::: "memory");

    int nodes = p.tree_lens ? p.tree_lens[b] : p.tree_tokens;
    if (nodes < 0 || nodes > p.tree_tokens) {
        if (t == 0 && rank == 0 && threadIdx.x == 0 && p.status) atomicOr(p.status, kFlagTreeRange);
        nodes = 0;
    }
    const bool live = t < nodes;                              // (the same for the whole cluster)
    const int first = rank * p.slice, here = max(0, min(p.slice, p.vocab - first));
    const E *from = static_cast<const E *>(p.logits) + row * p.row_stride + first;
    const int words = (p.vocab + 31) / 32;
    const uint32_t *allowed = p.allowed ? p.allowed + row * words : nullptr;

    float z[kGroups][kVec];
    if (live) {
#pragma unroll
        for (int g = 0; g < kGroups; ++g) {
            const int at = (g * kLogitThreads + threadIdx.x) * kVec;
            if (at + kVec <= here) {
                logit_load<E, kVec>(from + at, z[g]);
            } else {
#pragma unroll
                for (int i = 0; i < kVec; ++i) z[g][i] = at + i < here ? logit_value(from[at + i]) : -INFINITY;
            }
        }
    }

    // ---- what was said, while the logits are on their way ----
    const bool counts = live && p.penalties != nullptr, biased = live && p.bias_tokens != nullptr && p.max_bias > 0;
    float repetition = 1.f, frequency = 0.f, presence = 0.f;
    if (counts || biased) {
        for (int i = threadIdx.x; i < (here + 3) / 4; i += kLogitThreads) reinterpret_cast<uint4 *>(table)[i] = make_uint4(0u, 0u, 0u, 0u);
        __syncthreads();
        bool bad = false;
        auto note = [&](int token, unsigned what, bool count) {
            if (token < 0 || token >= p.vocab) {
                bad = true;
                return;
            }
            const int at = token - first;
            if (at < 0 || at >= here) return;
            if (count) atomicAdd(table + at, what);
            else atomicOr(table + at, what);
        };
        if (counts) {
            repetition = p.penalties[(int64_t)b * 3];
            frequency = p.penalties[(int64_t)b * 3 + 1];
            presence = p.penalties[(int64_t)b * 3 + 2];
            if (p.tokens) {
                int len = p.token_lens ? p.token_lens[b] : p.max_tokens, prompt = p.prompt_lens ? p.prompt_lens[b] : 0;
                if (len < 0 || len > p.max_tokens || prompt < 0 || prompt > len) {
                    bad = true;
                    len = prompt = 0;
                }
                const int32_t *said = p.tokens + (int64_t)b * p.max_tokens;
                constexpr int kDeep = 4;
                for (int i0 = threadIdx.x; i0 < len; i0 += kDeep * kLogitThreads) {
                    int token[kDeep];
#pragma unroll
                    for (int u = 0; u < kDeep; ++u) token[u] = i0 + u * kLogitThreads < len ? said[i0 + u * kLogitThreads] : 0;
#pragma unroll
                    for (int u = 0; u < kDeep; ++u) {
                        const int i = i0 + u * kLogitThreads;
                        if (i < len) note(token[u], i < prompt ? kLogitPrompted : 1u, i >= prompt);
                    }
                }
            }
            if (p.draft_tokens && threadIdx.x < nodes) {
                const int j = threadIdx.x;
                bool sees = j <= t;
                if (p.tree_mask) sees = p.tree_mask[row * ((p.tree_tokens + 63) / 64) + j / 64] >> (j & 63) & 1u;
                if (sees) note(p.draft_tokens[(int64_t)b * p.tree_tokens + j], 1u, true);
            }
        }
        if (biased && threadIdx.x < p.max_bias) {
            const int token = p.bias_tokens[(int64_t)b * p.max_bias + threadIdx.x];
            bias_tokens[threadIdx.x] = token;
            bias_values[threadIdx.x] = p.bias_values[(int64_t)b * p.max_bias + threadIdx.x];
            if (token >= 0) note(token, kLogitBiased, false);                 // (negative: an unused entry)
        }
        if (bad && rank == 0 && p.status) atomicOr(p.status, kFlagTokenRange);
        __syncthreads();
    }

    // ---- penalties, biases, mask; the largest ----
    const float temperature = p.temperatures ? p.temperatures[b] : 1.f;
    LogitBest best = {-INFINITY, INT32_MAX};
    if (live) {
#pragma unroll
        for (int g = 0; g < kGroups; ++g) {
            const int at = (g * kLogitThreads + threadIdx.x) * kVec;
            if (at >= here) continue;
            unsigned said[kVec] = {};
            if (counts || biased) {
                if constexpr (kVec == 4) *reinterpret_cast<uint4 *>(said) = *reinterpret_cast<const uint4 *>(table + at);
                else said[0] = table[at];
            }
            const unsigned may = allowed ? allowed[(first + at) >> 5] >> ((first + at) & 31) : ~0u;
#pragma unroll
            for (int i = 0; i < kVec; ++i) {
                float x = z[g][i];
                if (said[i] != 0) {
                    const unsigned n = said[i] & (kLogitBiased - 1u);
                    if (said[i] & (kLogitPrompted | (kLogitBiased - 1u))) {
                        x = x > 0.f ? x / repetition : x * repetition;
                        x = x - frequency * (float)n - (n > 0 ? presence : 0.f);
                    }
                    if (said[i] & kLogitBiased) {
                        float sum = 0.f;
                        for (int j = 0; j < p.max_bias; ++j)
                            if (bias_tokens[j] == first + at + i) sum += bias_values[j];
                        x += sum;
                    }
                }
                if (!(may >> i & 1u) || at + i >= here) x = -INFINITY;
                z[g][i] = x;
                best.take(x, first + at + i);
            }
        }
    }
    const int type = p.out_type;
    const int64_t to = row * p.out_stride + first;
    if (!p.probabilities) {
        if (live) {
#pragma unroll
            for (int g = 0; g < kGroups; ++g) {
                const int at = (g * kLogitThreads + threadIdx.x) * kVec;
                if (at >= here) continue;
                if (temperature > 0.f) {
#pragma unroll
                    for (int i = 0; i < kVec; ++i) z[g][i] = z[g][i] / temperature;
                }
                logit_store<kVec>(p.out, type, to + at, z[g], min(kVec, here - at));
            }
        }
        asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
        return;
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) best.take(__shfl_xor_sync(0xffffffffu, best.value, o), __shfl_xor_sync(0xffffffffu, best.at, o));
    if (lane == 0) best_by_warp[warp] = best;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kLogitWarps; ++w) best.take(best_by_warp[w].value, best_by_warp[w].at);

    // ---- exponentials against the block's own maximum, and their sum ----
    const bool greedy = !(temperature > 0.f);
    const float rate = greedy ? 0.f : fminf(1.44269504088896340736f / temperature, 1e30f);
    const float top = best.value == -INFINITY ? 0.f : best.value;             // (nothing is left: all exponentials are 0)
    float sum = 0.f;
    if (live && !greedy) {
#pragma unroll
        for (int g = 0; g < kGroups; ++g) {
#pragma unroll
            for (int i = 0; i < kVec; ++i) {
                const bool is = (g * kLogitThreads + threadIdx.x) * kVec + i < here;
                z[g][i] = is ? fast_exp2((z[g][i] - top) * rate) : 0.f;
                sum += z[g][i];
            }
        }
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    if (lane == 0) sum_by_warp[warp] = sum;
    __syncthreads();
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");       // every block of the cluster has begun
    if (threadIdx.x < ctas) {
        float total = 0.f;
#pragma unroll
        for (int w = 0; w < kLogitWarps; ++w) total += sum_by_warp[w];
        cluster.map_shared_rank(best_by_cta, threadIdx.x)[rank] = best;
        cluster.map_shared_rank(sum_by_cta, threadIdx.x)[rank] = total;
    }
    cluster.sync();
    if (!live) return;
    LogitBest all = best_by_cta[0];
    for (int c = 1; c < ctas; ++c) all.take(best_by_cta[c].value, best_by_cta[c].at);
    const float all_top = all.value == -INFINITY ? 0.f : all.value;
    float total = 0.f;
    for (int c = 0; c < ctas; ++c) {
        const float its = best_by_cta[c].value == -INFINITY ? 0.f : best_by_cta[c].value;
        if (sum_by_cta[c] != 0.f) total += sum_by_cta[c] * (its == all_top ? 1.f : fast_exp2((its - all_top) * rate));
    }
    const float factor = (top == all_top ? 1.f : fast_exp2((top - all_top) * rate)) / (total == 0.f ? 1.f : total);
#pragma unroll
    for (int g = 0; g < kGroups; ++g) {
        const int at = (g * kLogitThreads + threadIdx.x) * kVec;
        if (at >= here) continue;
#pragma unroll
        for (int i = 0; i < kVec; ++i)
            z[g][i] = greedy ? (first + at + i == all.at && all.value != -INFINITY ? 1.f : 0.f) : sum_by_cta[rank] == 0.f && total == total ? 0.f : z[g][i] * factor;
        logit_store<kVec>(p.out, type, to + at, z[g], min(kVec, here - at));
    }
}

}  // namespace instinfer
