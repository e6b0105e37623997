// Rotary positions on the way into the cache, for sm_100a: the new tokens' queries and keys are turned, and the
// keys and values (or latent rows) join the cache in the same pass.
//
// A pair (a, b) of a head's dims at position p becomes m (a cos t - b sin t, a sin t + b cos t), t = p f_i with f_i the
// frequency of pair i.  Far positions turn fast pairs by 10^5 radians and more, where a product in 32 bits is off by
// hundredths of a radian: the angle is taken in 64 bits, reduced to a fraction of a turn there, and only its sine and
// cosine are 32-bit numbers.  They are the same for every head of a token, so a block makes them once for its tokens
// and turns all (or, where tokens are few, some) of their heads by them.
//
// Bound by bytes: every value is read once and written once, 16 bytes a thread and access.  A unit is 16 dims of a
// head (two octets): the two halves' partners in the half layout, neighbours in the interleaved one, so that a pair
// never leaves its thread.  A thread's first units are asked for before its block knows the tokens' lengths and pages.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "decode_attention_kernels.cuh"

namespace instinfer {

constexpr int kRopeThreads = 256;
constexpr int kRopeTokens = 4;          // tokens of a block at most
constexpr int kRopeMaxPairs = 128;      // rotary dims of a head / 2
constexpr int kRopeUnits = 2;           // units that a thread has in flight

struct RopeParams {
    const void *q;                // token n's heads at n * q_stride elements, q_head_stride apart
    const void *k;                // latent form: the shared key part, one head of rope dims
    const void *v;                // latent form: the latent row, v_units units
    void *q_out;                  // token n's heads at n * q_out_stride, q_out_head_stride apart, the turned dims first
    void *k_cache;                // latent form: the latent cache
    void *v_cache;
    const double *frequencies;    // [pairs] radians per position
    const int32_t *positions;     // nullable [batch, max_new]
    const int32_t *seq_lens;
    const int32_t *new_lens;      // nullable: max_new each
    const int32_t *block_table;   // nullptr: contiguous
    int32_t *status;
    int64_t q_stride, k_stride, v_stride, q_head_stride;
    int64_t q_out_stride, q_out_head_stride;
    int64_t num_phys_blocks;
    int64_t cache_rows;           // rows of a cache that the call's shapes imply
    int32_t batch, max_new;
    int32_t q_heads, kv_heads;
    int32_t head_units;           // units of a q or k head: head_dim / 16 (latent form: of the turned part)
    int32_t v_units;              // of a v head (latent form: of the latent vector)
    int32_t pairs;                // turned dims / 2
    int32_t s_max, block_tokens, max_blocks_per_seq;
    int32_t tokens_per_block;     // 1 .. kRopeTokens
    int32_t parts;                // blocks that share a token's units
    float magnitude;
};

// Eight values as they lie in memory.
template <typename E>
struct RopeOctet {
    uint4 raw[sizeof(E) / 2];
    __device__ __forceinline__ void load(const E *from)
    {
#pragma unroll
        for (int i = 0; i < (int)sizeof(E) / 2; ++i) raw[i] = reinterpret_cast<const uint4 *>(from)[i];
    }
    __device__ __forceinline__ void values(float (&x)[8]) const
    {
        const unsigned *w = reinterpret_cast<const unsigned *>(raw);
        if constexpr (sizeof(E) == 4) {
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = __uint_as_float(w[i]);
        } else if constexpr (sizeof(E) == 2) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                float2 two;
                if constexpr (__is_same(E, __half)) two = __half22float2(*reinterpret_cast<const __half2 *>(&w[i]));
                else two = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162 *>(&w[i]));
                x[2 * i] = two.x;
                x[2 * i + 1] = two.y;
            }
        }
    }
};
template <typename E>
__device__ __forceinline__ uint4 rope_pack(const float (&x)[8])
{
    unsigned w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (__is_same(E, __half)) {
            const __half2 two = __floats2half2_rn(x[2 * i], x[2 * i + 1]);
            w[i] = *reinterpret_cast<const unsigned *>(&two);
        } else {
            const __nv_bfloat162 two = __floats2bfloat162_rn(x[2 * i], x[2 * i + 1]);
            w[i] = *reinterpret_cast<const unsigned *>(&two);
        }
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}
// An octet that is not turned: its bits where the types are alike, else rounded once.
template <typename In, typename Out>
__device__ __forceinline__ uint4 rope_copy(const RopeOctet<In> &x)
{
    if constexpr (__is_same(In, Out)) {
        return x.raw[0];
    } else {
        float v[8];
        x.values(v);
        return rope_pack<Out>(v);
    }
}

// kLatent: the cache is one row a token, the latent vector and behind it the turned key part, and the queries' turned
// part is written into the rows of the absorbed queries.  Otherwise K and V caches [.., heads, tokens, head_dim].
template <typename In, typename Out, bool kInterleaved, bool kLatent>
__global__ void __launch_bounds__(kRopeThreads)
rope_append_kernel(const RopeParams p)
{
    struct Token {
        int64_t row;              // of the cache (K and V: of its block's or sequence's first head)
        double position;
        int live, writable;       // a new token; one whose cache row exists
    };
    __shared__ Token tokens[kRopeTokens];
    __shared__ float2 turns[kRopeTokens * kRopeMaxPairs];

    const int part = blockIdx.x % p.parts;
    const int64_t n0 = (int64_t)(blockIdx.x / p.parts) * p.tokens_per_block, all = (int64_t)p.batch * p.max_new;
    const int here = (int)(all - n0 < p.tokens_per_block ? all - n0 : p.tokens_per_block);
    const int q_units = p.q_heads * p.head_units, k_units = p.kv_heads * p.head_units;
    const int units = q_units + k_units + (kLatent ? p.v_units : p.kv_heads * p.v_units);
    // (a token's units are dealt to its parts in turn, so that a warp's stay neighbours)
    const int mine = (units - part * kRopeThreads + p.parts * kRopeThreads - 1) / (p.parts * kRopeThreads);    // rounds of kRopeThreads units per token
    const int rounds = mine > 0 ? mine * here : 0;
    asm volatile("griddepcontrol.launch_dependents;");      // the next kernel may start being scheduled
    asm volatile("griddepcontrol.wait;" ::: "memory");      // earlier kernels' writes are visible from here

    struct Unit {
        RopeOctet<In> first, second;
        int token, unit;          // unit < 0: none
    };
    Unit units_now[kRopeUnits];
    // The two octets of unit j of a q or k head of p.head_units units: partners where they are turned.
    auto octets = [&](int j, int &first, int &second) {
        first = 16 * j;
        second = first + 8;
        if (!kInterleaved && j < p.pairs / 8) {
            first = 8 * j;
            second = p.pairs + first;
        }
    };
    auto ask = [&](int round, Unit &u) {
        u.unit = -1;
        if (round >= rounds) return;
        u.token = round / mine;
        const int unit = ((round - u.token * mine) * p.parts + part) * kRopeThreads + threadIdx.x;
        if (unit >= units) return;
        u.unit = unit;
        const int64_t n = n0 + u.token;
        const In *from;
        int a, b;
        if (unit < q_units) {
            const int head = unit / p.head_units;
            from = static_cast<const In *>(p.q) + n * p.q_stride + head * p.q_head_stride;
            octets(unit - head * p.head_units, a, b);
        } else if (unit < q_units + k_units) {
            const int head = (unit - q_units) / p.head_units;
            from = static_cast<const In *>(p.k) + n * p.k_stride + head * (p.head_units * 16);
            octets(unit - q_units - head * p.head_units, a, b);
        } else {
            from = static_cast<const In *>(p.v) + n * p.v_stride;
            a = (unit - q_units - k_units) * 16;
            b = a + 8;
        }
        u.first.load(from + a);
        u.second.load(from + b);
    };
#pragma unroll
    for (int i = 0; i < kRopeUnits; ++i) ask(i, units_now[i]);

    if (threadIdx.x < here) {
        const int64_t n = n0 + threadIdx.x;
        const int b = (int)(n / p.max_new), t = (int)(n - (int64_t)b * p.max_new);
        Token token = {0, 0.0, 0, 0};
        const int len = p.seq_lens[b];
        const int fresh = p.new_lens ? p.new_lens[b] : len == 0 ? 0 : p.max_new;
        const int64_t capacity = p.block_table ? (int64_t)p.max_blocks_per_seq * p.block_tokens : (int64_t)p.s_max;
        if (len < 0 || len > capacity || fresh < 0 || fresh > p.max_new || fresh > len) {
            if (t == 0 && part == 0 && p.status) atomicOr(p.status, 1);          // lengths out of range: sequence skipped
        } else if (t < fresh) {
            const int at = len - fresh + t;
            token.live = token.writable = 1;
            token.position = p.positions ? p.positions[n] : at;
            if (p.block_table) {
                const int phys = p.block_table[(int64_t)b * p.max_blocks_per_seq + at / p.block_tokens];
                if (phys < 0 || (int64_t)phys >= p.num_phys_blocks) {
                    if (part == 0 && p.status) atomicOr(p.status, 2);            // rows of a bad block are skipped
                    token.writable = 0;
                } else {
                    token.row = (int64_t)phys * p.block_tokens * (kLatent ? 1 : p.kv_heads) + at % p.block_tokens;
                }
            } else {
                token.row = (int64_t)b * p.s_max * (kLatent ? 1 : p.kv_heads) + at;
            }
        }
        tokens[threadIdx.x] = token;
    }
    // (frequencies come from far; the first one is asked for before the wait)
    const double frequency = threadIdx.x < here * p.pairs ? p.frequencies[threadIdx.x % p.pairs] : 0.0;
    __syncthreads();
    for (int i = threadIdx.x; i < here * p.pairs; i += kRopeThreads) {
        const int token = i / p.pairs;
        const double f = i < kRopeThreads ? frequency : p.frequencies[i - token * p.pairs];
        const double part_of_turn = tokens[token].position * f * 0.15915494309189533577;
        float sine, cosine;
        sincospif(2.f * (float)(part_of_turn - rint(part_of_turn)), &sine, &cosine);
        turns[i] = make_float2(cosine * p.magnitude, sine * p.magnitude);
    }
    __syncthreads();

    auto finish = [&](const Unit &u) {
        if (u.unit < 0) return;
        const Token &token = tokens[u.token];
        if (!token.live) return;
        const int64_t n = n0 + u.token;
        const bool is_q = u.unit < q_units, is_v = u.unit >= q_units + k_units;
        const int inside = is_q ? u.unit : is_v ? u.unit - q_units - k_units : u.unit - q_units;
        const int per_head = is_v ? p.v_units : p.head_units, head = inside / per_head, j = inside - head * per_head;
        int a = 16 * j, b = a + 8;
        if (!is_v) octets(j, a, b);
        uint4 x, y;
        if (!is_v && j < p.pairs / 8) {
            float first[8], second[8], new_first[8], new_second[8];
            u.first.values(first);
            u.second.values(second);
            const float2 *turn = turns + u.token * p.pairs + 8 * j;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                if constexpr (kInterleaved) {
                    // pairs (0, 1), (2, 3) .. of each octet
                    const float re = i < 4 ? first[(2 * i) & 7] : second[(2 * i) & 7], im = i < 4 ? first[(2 * i + 1) & 7] : second[(2 * i + 1) & 7];
                    const float new_re = re * turn[i].x - im * turn[i].y, new_im = re * turn[i].y + im * turn[i].x;
                    if (i < 4) {
                        new_first[(2 * i) & 7] = new_re;
                        new_first[(2 * i + 1) & 7] = new_im;
                    } else {
                        new_second[(2 * i) & 7] = new_re;
                        new_second[(2 * i + 1) & 7] = new_im;
                    }
                } else {
                    new_first[i] = first[i] * turn[i].x - second[i] * turn[i].y;
                    new_second[i] = first[i] * turn[i].y + second[i] * turn[i].x;
                }
            }
            x = rope_pack<Out>(new_first);
            y = rope_pack<Out>(new_second);
        } else {
            x = rope_copy<In, Out>(u.first);
            y = rope_copy<In, Out>(u.second);
        }
        Out *to;
        if (is_q) {
            to = static_cast<Out *>(p.q_out) + n * p.q_out_stride + head * p.q_out_head_stride;
        } else {
            if (!token.writable) return;
            if constexpr (kLatent) {
                const int row_dims = p.v_units * 16 + p.head_units * 16;
                if (!bounds_ok(token.row >= 0 && token.row < p.cache_rows, p.status)) return;
                to = static_cast<Out *>(p.k_cache) + token.row * row_dims + (is_v ? 0 : p.v_units * 16);
            } else {
                const int64_t row = token.row + (int64_t)head * (p.block_table ? p.block_tokens : p.s_max);
                if (!bounds_ok(row >= 0 && row < p.cache_rows, p.status)) return;
                to = static_cast<Out *>(is_v ? p.v_cache : p.k_cache) + row * (p.head_units * 16);
            }
        }
        *reinterpret_cast<uint4 *>(to + a) = x;
        *reinterpret_cast<uint4 *>(to + b) = y;
    };
    for (int round = 0; round < rounds; round += kRopeUnits) {
#pragma unroll
        for (int i = 0; i < kRopeUnits; ++i) finish(units_now[i]);
        if (round + kRopeUnits < rounds) {
#pragma unroll
            for (int i = 0; i < kRopeUnits; ++i) ask(round + kRopeUnits + i, units_now[i]);
        }
    }
}

}  // namespace instinfer
