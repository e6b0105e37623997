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
// maximum and the place of the maximum, once, by stores that count their bytes at the receiver's barrier.
//
// The grid is as many clusters as the GPU holds at once, each with a run of consecutive rows, and rows of one tree share the
// table but for their own drafts.  Logits are asked for without a branch between the loads, and what sticks out of a row at
// its ends is kept out of the loops over all of it.  Measured: one row of 32,000 fp32 5.8 us; 192 rows of 50,257 bf16 with
// everything on 65 to 76 us and 512 rows of 131,072 in trees 251 to 262 us, six to eight times what their bytes take.  The softmax
// alone is 38 and 163 us of them: two blocks of 512 threads per SM wait together at each of a row's steps with nothing of the
// next row under way, and leave a thread 64 registers, so that the instance with 32 logits a thread spills (234 bytes of stores
// and 306 of loads).  History and drafts add 20 and 75 us, biases 4, the grammar 3 and 15.
#pragma once

#include <cooperative_groups.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include <type_traits>

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
    int32_t rows, tree_tokens, vocab;
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
// kVec (1 or 4) logits as they lie in memory.
template <typename E, int kVec>
struct LogitRaw {
    using Word = typename std::conditional<kVec == 1, E, typename std::conditional<sizeof(E) == 4, float4, uint2>::type>::type;
    Word word;
    __device__ __forceinline__ void nothing()                 // -infinities
    {
        const E one = E(-INFINITY);
#pragma unroll
        for (int i = 0; i < kVec; ++i) reinterpret_cast<E *>(&word)[i] = one;
    }
    __device__ __forceinline__ void values(float (&x)[kVec]) const
    {
        const E *one = reinterpret_cast<const E *>(&word);
#pragma unroll
        for (int i = 0; i < kVec; ++i) x[i] = logit_value(one[i]);
    }
};
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
template <typename Out, int kVec>
__device__ __forceinline__ void logit_store(Out *to, const float (&x)[kVec])
{
    if constexpr (kVec == 1) {
        if constexpr (sizeof(Out) == 4) to[0] = x[0];
        else if constexpr (std::is_same<Out, __half>::value) to[0] = __float2half_rn(x[0]);
        else to[0] = __float2bfloat16_rn(x[0]);
    } else if constexpr (sizeof(Out) == 4) {
        *reinterpret_cast<float4 *>(to) = make_float4(x[0], x[1], x[2], x[3]);
    } else {
        *reinterpret_cast<uint2 *>(to) = make_uint2(logit_pack<Out>(x[0], x[1]), logit_pack<Out>(x[2], x[3]));
    }
}
static __device__ __noinline__ void logit_store_one(void *out, int type, int64_t at, float x)
{
    const float one[1] = {x};
    if (type == 0) logit_store<float, 1>(static_cast<float *>(out) + at, one);
    else if (type == 1) logit_store<__half, 1>(static_cast<__half *>(out) + at, one);
    else logit_store<__nv_bfloat16, 1>(static_cast<__nv_bfloat16 *>(out) + at, one);
}

// 2^x, with 0 for what would be subnormal: two instructions fewer for every logit.
__device__ __forceinline__ float logit_exp2(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// What a block knows of its part of a row: the largest, the sum of exponentials against it, its first place.
struct __align__(16) LogitShare {
    float top, sum;
    int place, pad;
};
// Stores a share at the same place of block `to` of the cluster and reports its bytes to the same barrier there.
__device__ __forceinline__ void logit_send(unsigned at, unsigned bar, int to, const LogitShare &share)
{
    unsigned there, bar_there;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(there) : "r"(at), "r"(to));
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(bar_there) : "r"(bar), "r"(to));
    asm volatile("st.async.shared::cluster.mbarrier::complete_tx::bytes.v4.b32 [%0], {%1, %2, %3, %4}, [%5];"
                 :: "r"(there), "r"(__float_as_uint(share.top)), "r"(__float_as_uint(share.sum)), "r"(share.place), "r"(0), "r"(bar_there) : "memory");
}

// The sequence's biases of one token, in the list's order.
static __device__ __noinline__ float logit_bias(const int *tokens, const float *values, int n, int token)
{
    float sum = 0.f;
    for (int j = 0; j < n; ++j)
        if (tokens[j] == token) sum += values[j];
    return sum;
}

// kHeld: logits of a thread; kVec: how many of them lie together (4 where input and output rows start alike between 16-byte
// boundaries, which an odd vocabulary's rows do: the row's first group then begins up to three tokens before it).
template <typename E, int kHeld, int kVec>
__global__ void __launch_bounds__(kLogitThreads, kVec == 4 && kHeld <= 32 ? 2 : 1)
process_logits_kernel(const LogitParams p)
{
    namespace cg = cooperative_groups;
    constexpr int kGroups = kHeld / kVec;
    using Bits = typename std::conditional<(kHeld > 32), uint64_t, uint32_t>::type;       // one of every held token
    extern __shared__ __align__(16) unsigned table[];         // [slice], where there is anything to look up
    __shared__ float top_by_warp[kLogitWarps], sum_by_warp[kLogitWarps];
    __shared__ LogitShare by_cta[2][kLogitMaxCtas];
    __shared__ uint64_t arrived[2];                           // mbarriers: all blocks' shares of a row are here
    __shared__ int first_place[2];
    __shared__ int bias_tokens[kLogitMaxBias];
    __shared__ float bias_values[kLogitMaxBias];
    const cg::cluster_group cluster = cg::this_cluster();
    const int ctas = (int)cluster.num_blocks(), rank = (int)cluster.block_rank();
    const int clusters = gridDim.x / ctas, mine = blockIdx.x / ctas;
    const int64_t row0 = (int64_t)p.rows * mine / clusters, row1 = (int64_t)p.rows * (mine + 1) / clusters;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int words = (p.vocab + 31) / 32, type = p.out_type;
    const bool counts = p.penalties != nullptr, biased = p.bias_tokens != nullptr && p.max_bias > 0;
    asm volatile("griddepcontrol.launch_dependents;");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    if (ctas > 1) {
        if (threadIdx.x < 2) mbarrier_init(static_cast<unsigned>(__cvta_generic_to_shared(arrived + threadIdx.x)), 1);
        mbarrier_init_fence();
        cluster.sync();                                       // (a block writes to another one's memory only once that has begun)
    }

    // What the table is made for: a sequence's history and biases, on places that start at `first` of its row.
    int table_b = -1, table_shift = 0, noted = -1;            // noted: the place where this thread counted a draft
    float repetition = 1.f, frequency = 0.f, presence = 0.f;
    // Which exchange buffers, and the phase of their barrier.  (Two: a block that is a row ahead writes to the others.  It is
    // never two ahead, since it waits for their shares of the row between.)
    int turn = 0;
    unsigned phase = 0;
    for (int64_t row = row0; row < row1; ++row) {
        const int b = (int)(row / p.tree_tokens), t = (int)(row - (int64_t)b * p.tree_tokens);
        int nodes = p.tree_lens ? p.tree_lens[b] : p.tree_tokens;
        if (nodes < 0 || nodes > p.tree_tokens) {
            if (t == 0 && rank == 0 && threadIdx.x == 0 && p.status) atomicOr(p.status, kFlagTreeRange);
            nodes = 0;
        }
        if (t >= nodes) continue;                             // (the same for the whole cluster)
        // Token of place 0 of this block's slice (negative: places before the row are nobody's), and places up to the row's end.
        const int shift = kVec == 1 ? 0 : (int)(row * p.row_stride & (kVec - 1)), first = rank * p.slice - shift;
        const int here = max(0, min(p.slice, p.vocab - first));
        const E *from = static_cast<const E *>(p.logits) + row * p.row_stride + first;
        auto place = [&](int g) -> int { return (g * kLogitThreads + threadIdx.x) * kVec; };
        // Whether n places from `at` on are the row's, and the block's (looked at in the bounds-checking build only).
        auto inside = [&](int at, int n) -> bool {
            return bounds_ok(at >= 0 && at + n <= p.slice && first + at >= 0 && first + at + n <= p.vocab, p.status);
        };
        // Places [lead, here) are the row's; a group of kVec places may stick out at either end.
        const int lead = rank == 0 ? shift : 0, last = here - kVec;
        const bool ragged = lead != 0 || here % kVec != 0;    // (the same for the block: what sticks out is kept out of the loops over all)

        // All that comes from memory is asked for at once.
        const bool fresh = (counts || biased) && (b != table_b || shift != table_shift);
        int said_len = 0, prompt = 0;
        if (fresh && counts && p.tokens) {
            said_len = p.token_lens ? p.token_lens[b] : p.max_tokens;
            prompt = p.prompt_lens ? p.prompt_lens[b] : 0;
        }
        const float temperature = p.temperatures ? p.temperatures[b] : 1.f;
        // (no branch between the loads and no use before the last of them, so that they are all under way together)
        LogitRaw<E, kVec> raw[kGroups];
#pragma unroll
        for (int g = 0; g < kGroups; ++g) {
            const int at = place(g);
            raw[g].nothing();
            if (at >= lead && at <= last && inside(at, kVec)) raw[g].word = *reinterpret_cast<const typename LogitRaw<E, kVec>::Word *>(from + at);
        }
        Bits may = 0;                                         // bit g * kVec + i: the token is allowed
        if (p.allowed) {
            const uint32_t *allowed = p.allowed + row * words;
            uint32_t low[kGroups];
#pragma unroll
            for (int g = 0; g < kGroups; ++g) low[g] = place(g) < here ? allowed[max(first + place(g), 0) >> 5] : 0u;
#pragma unroll
            for (int g = 0; g < kGroups; ++g) {
                const int token = first + place(g);
                unsigned bits = token < 0 ? low[g] << -token : low[g] >> (token & 31);
                // (a group's bits may lie in two words where the row begins late)
                if (kVec > 1 && shift != 0 && place(g) < here && (token & 31) > 32 - kVec && (token >> 5) + 1 < words)
                    bits |= allowed[(token >> 5) + 1] << (32 - (token & 31));
                may |= (Bits)(bits & ((1u << kVec) - 1)) << (g * kVec);
            }
        }
        float z[kGroups][kVec];
#pragma unroll
        for (int g = 0; g < kGroups; ++g) raw[g].values(z[g]);
        if (ragged) {
#pragma unroll
            for (int g = 0; g < kGroups; ++g) {
                const int at = place(g);
#pragma unroll
                for (int i = 0; i < kVec; ++i)
                    if (!(at >= lead && at <= last) && at + i < here && at + i >= lead && inside(at + i, 1)) z[g][i] = logit_value(from[at + i]);
            }
        }

        // ---- what was said, while the logits are on their way ----
        if (counts || biased) {
            bool bad = false;
            // Counts `what` for a token of this block's places; the place, or -1.
            auto note = [&](int which, unsigned what, bool count) -> int {
                if (which < 0 || which >= p.vocab) {
                    bad = true;
                    return -1;
                }
                const int at = which - first;
                if (at < 0 || at >= here || !inside(at, 1)) return -1;
                if (count) atomicAdd(table + at, what);
                else atomicOr(table + at, what);
                return at;
            };
            int draft = -1;                                   // of the nodes that this one sees, one a thread
            bool drafted = false;
            if (counts && p.draft_tokens && threadIdx.x < nodes) {
                const int j = threadIdx.x;
                drafted = p.tree_mask ? (p.tree_mask[row * ((p.tree_tokens + 63) / 64) + j / 64] >> (j & 63) & 1u) != 0 : j <= t;
                if (drafted) draft = p.draft_tokens[(int64_t)b * p.tree_tokens + j];
            }
            if (fresh) {
                if (said_len < 0 || said_len > p.max_tokens || prompt < 0 || prompt > said_len) {
                    bad = true;
                    said_len = prompt = 0;
                }
                if (counts) {
                    repetition = p.penalties[(int64_t)b * 3];
                    frequency = p.penalties[(int64_t)b * 3 + 1];
                    presence = p.penalties[(int64_t)b * 3 + 2];
                }
                constexpr int kDeep = 4;
                const int32_t *said = p.tokens + (int64_t)b * p.max_tokens;
                int token[kDeep];
                auto ask = [&](int i0) {
#pragma unroll
                    for (int u = 0; u < kDeep; ++u) token[u] = i0 + u * kLogitThreads < said_len ? said[i0 + u * kLogitThreads] : 0;
                };
                ask(threadIdx.x);
                __syncthreads();                              // (the last row has read the table and the biases)
                int bias_token = -1;
                if (biased && threadIdx.x < p.max_bias) {
                    bias_token = p.bias_tokens[(int64_t)b * p.max_bias + threadIdx.x];
                    bias_tokens[threadIdx.x] = bias_token;
                    bias_values[threadIdx.x] = p.bias_values[(int64_t)b * p.max_bias + threadIdx.x];
                }
                for (int i = threadIdx.x; i < (here + 3) / 4; i += kLogitThreads) reinterpret_cast<uint4 *>(table)[i] = make_uint4(0u, 0u, 0u, 0u);
                __syncthreads();
                for (int i0 = threadIdx.x; i0 < said_len; i0 += kDeep * kLogitThreads) {
                    int now[kDeep];
#pragma unroll
                    for (int u = 0; u < kDeep; ++u) now[u] = token[u];
                    ask(i0 + kDeep * kLogitThreads);
#pragma unroll
                    for (int u = 0; u < kDeep; ++u) {
                        const int i = i0 + u * kLogitThreads;
                        if (i < said_len) (void)note(now[u], i < prompt ? kLogitPrompted : 1u, i >= prompt);
                    }
                }
                if (bias_token >= 0) (void)note(bias_token, kLogitBiased, false);         // (negative: an unused entry)
                table_b = b;
                table_shift = shift;
                noted = -1;
            }
            // (The table of another node of the same tree: its drafts go, this node's come.  A barrier lies between the last
            // row's look-ups and here.)
            if (noted >= 0) atomicSub(table + noted, 1u);
            noted = drafted ? note(draft, 1u, true) : -1;
            if (bad && rank == 0 && p.status) atomicOr(p.status, kFlagTokenRange);
            __syncthreads();
        }

        // ---- penalties, biases, mask; the largest ----
        float top = -INFINITY;
#pragma unroll
        for (int g = 0; g < kGroups; ++g) {
            const int at = place(g);
            if ((counts || biased) && at < here) {
                unsigned said[kVec];
                if constexpr (kVec == 4) *reinterpret_cast<uint4 *>(said) = *reinterpret_cast<const uint4 *>(table + at);
                else said[0] = table[at];
                unsigned any = said[0];
#pragma unroll
                for (int i = 1; i < kVec; ++i) any |= said[i];
                if (any != 0) {                               // (rare)
#pragma unroll
                    for (int i = 0; i < kVec; ++i) {
                        float x = z[g][i];
                        const unsigned n = said[i] & (kLogitBiased - 1u);
                        if (said[i] & (kLogitPrompted | (kLogitBiased - 1u))) {
                            x = x > 0.f ? x / repetition : x * repetition;
                            x = x - frequency * (float)n - (n > 0 ? presence : 0.f);
                        }
                        if (said[i] & kLogitBiased) x += logit_bias(bias_tokens, bias_values, p.max_bias, first + at + i);
                        z[g][i] = x;
                    }
                }
            }
            if (p.allowed) {
#pragma unroll
                for (int i = 0; i < kVec; ++i)
                    if (!(may >> (g * kVec + i) & 1u)) z[g][i] = -INFINITY;
            }
#pragma unroll
            for (int i = 0; i < kVec; ++i) top = fmaxf(top, z[g][i]);
        }
        const int64_t to = row * p.out_stride + first;
        // Writes the groups, times a factor; of a group that sticks out of the row, what belongs to it.
        auto write = [&](auto kind, float times) {
            using Out = decltype(kind);
            Out *out = static_cast<Out *>(p.out) + to;
#pragma unroll
            for (int g = 0; g < kGroups; ++g) {
                const int at = place(g);
#pragma unroll
                for (int i = 0; i < kVec; ++i) z[g][i] *= times;
                if (at >= lead && at <= last && inside(at, kVec)) logit_store<Out, kVec>(out + at, z[g]);
            }
            if (ragged) {
#pragma unroll
                for (int g = 0; g < kGroups; ++g) {
                    const int at = place(g);
#pragma unroll
                    for (int i = 0; i < kVec; ++i)
                        if (!(at >= lead && at <= last) && at + i < here && at + i >= lead && inside(at + i, 1)) logit_store_one(p.out, type, to + at + i, z[g][i]);
                }
            }
        };
        auto write_all = [&](float times) {
            if (type == 0) write(float{}, times);
            else if (type == 1) write(__half{}, times);
            else write(__nv_bfloat16{}, times);
        };
        const bool greedy = !(temperature > 0.f);
        if (!p.probabilities) {
            if (!greedy) {
                // z / T rounded once, as the product with 1 / T in 64 bits: that is off by 2^-52 of itself, and a quotient of 24-bit
                // numbers is never within 2^-49 of itself of the middle between two of them.  (A division each takes 475 us for
                // 512 rows of 131,072; the product with a 32-bit inverse is rounded twice, and the inverse may overflow.)
                const double inverse = 1.0 / (double)temperature;
#pragma unroll
                for (int g = 0; g < kGroups; ++g) {
#pragma unroll
                    for (int i = 0; i < kVec; ++i) z[g][i] = (float)((double)z[g][i] * inverse);
                }
            }
            write_all(1.f);
            __syncthreads();                                  // (the table has been read)
            continue;
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
        if (lane == 0) top_by_warp[warp] = top;
        if (threadIdx.x == 0) first_place[turn] = INT32_MAX;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < kLogitWarps; ++w) top = fmaxf(top, top_by_warp[w]);

        // ---- exponentials against the block's own maximum, and their sum; or where the first of the largest is ----
        // (finite, so that the largest, 0 times it, keeps the exponent 0 at every temperature)
        const float rate = greedy ? 0.f : fminf(1.44269504088896340736f / temperature, 3.402823466e38f);
        float sum = 0.f;
        if (greedy) {
            int at = INT32_MAX;
#pragma unroll
            for (int g = 0; g < kGroups; ++g) {
#pragma unroll
                for (int i = 0; i < kVec; ++i)
                    if (z[g][i] == top) at = min(at, place(g) + i);
            }
            if (top > -INFINITY && at != INT32_MAX) atomicMin(first_place + turn, at);
        } else {
            // (The difference first: it is exact near the maximum, so that the blocks' sums join whatever their maxima.  As
            // 2^(rate z - rate top), in one instruction, the exponents are off by the rounding of rate top, another one in every
            // block and more than their whole range at small temperatures.)
            const float from_top = top == -INFINITY ? 0.f : top;              // (nothing is left: all exponentials are 0)
#pragma unroll
            for (int g = 0; g < kGroups; ++g) {
#pragma unroll
                for (int i = 0; i < kVec; ++i) {
                    z[g][i] = logit_exp2((z[g][i] - from_top) * rate);      // (0 where nothing is allowed)
                    sum += z[g][i];
                }
            }
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
        if (lane == 0) sum_by_warp[warp] = sum;
        __syncthreads();
        if (threadIdx.x < ctas) {
            float total = 0.f;
#pragma unroll
            for (int w = 0; w < kLogitWarps; ++w) total += sum_by_warp[w];
            const LogitShare share = {top, total, first_place[turn], 0};
            if (ctas > 1) {
                // Stored into block threadIdx.x, whose barrier counts the bytes: no fence, which would wait for the last row's output.
                const unsigned bar = static_cast<unsigned>(__cvta_generic_to_shared(arrived + turn));
                if (threadIdx.x == 0) mbarrier_expect_bytes(bar, ctas * (unsigned)sizeof(LogitShare));
                logit_send(static_cast<unsigned>(__cvta_generic_to_shared(&by_cta[turn][rank])), bar, threadIdx.x, share);
            } else {
                by_cta[turn][0] = share;
            }
        }
        if (ctas > 1) {
            if (!mbarrier_wait_bounded(static_cast<unsigned>(__cvta_generic_to_shared(arrived + turn)), phase)) {
                if (p.status) atomicOr(p.status, kFlagCopyTimeout);
                return;
            }
        } else {
            __syncthreads();
        }
        float all_top = -INFINITY;
        for (int c = 0; c < ctas; ++c) all_top = fmaxf(all_top, by_cta[turn][c].top);
        float total = 0.f;
        int winner = -1;                                      // the first block that has the largest
        for (int c = 0; c < ctas; ++c) {
            const float its = by_cta[turn][c].top, part = by_cta[turn][c].sum;
            if (winner < 0 && its == all_top && all_top > -INFINITY) winner = c;
            if (part != 0.f) total += part * (its == all_top ? 1.f : fast_exp2((its - all_top) * rate));
        }
        const int chosen = greedy && winner == rank ? by_cta[turn][rank].place : -1;
        // (a block that has nothing left gives zeros, unless the row is NaN)
        const float own = by_cta[turn][rank].sum, factor = own == 0.f && total == total ? 0.f : (top == all_top ? 1.f : fast_exp2((top - all_top) * rate)) / total;
        phase ^= (unsigned)turn;
        turn ^= 1;
        if (greedy) {
#pragma unroll
            for (int g = 0; g < kGroups; ++g) {
#pragma unroll
                for (int i = 0; i < kVec; ++i) z[g][i] = place(g) + i == chosen ? 1.f : 0.f;
            }
        }
        write_all(greedy ? 1.f : factor);
    }
}

}  // namespace instinfer
