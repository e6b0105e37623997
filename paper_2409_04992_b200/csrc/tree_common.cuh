// What the kernels that attend over a draft tree share, for sm_100a.
//
// A tree's nodes are the last tree_lens[b] positions of sequence b's cache.  A query row (a node's
// head) sees every position before them, and of the nodes those whose bits its mask row has.
#pragma once

#include "decode_attention_kernels.cuh"

namespace instinfer {

constexpr int kFlagTreeRange = 16;
constexpr int kMaxTreeTokens = 128;      // INSTINFER_MAX_TREE_TOKENS

struct TreeShape {
    const uint64_t *mask;          // [batch, tokens, words]
    const int32_t *lens;           // nullable: `tokens` each
    int32_t tokens;
    int32_t words;                 // 1 or 2
};

// The nodes that a row sees.
struct TreeRow {
    uint64_t lo, hi;               // nodes 0-63, 64-127
    bool all;                      // the row exists: it sees what lies before the tree
    // without the bits of nodes that a tree of `nodes` nodes does not have
    __device__ __forceinline__ TreeRow cut(int nodes) const
    {
        TreeRow row = *this;
        if (nodes < 64) row.lo &= ((uint64_t)1 << nodes) - 1;
        if (nodes <= 64) row.hi = 0;
        else if (nodes < 128) row.hi &= ((uint64_t)1 << (nodes - 64)) - 1;
        return row;
    }
    // node < 0: a position before the tree
    __device__ __forceinline__ bool sees(int node) const
    {
        if (node < 0) return all;
        return node < 128 && ((node < 64 ? lo : hi) >> (node & 63) & 1u) != 0;
    }
};

// Row `t` of sequence b's tree of `nodes` nodes; rows that are not nodes of it see nothing.
__device__ __forceinline__ TreeRow tree_row(const TreeShape &tree, int b, int t, int nodes)
{
    TreeRow row = {0, 0, false};
    if (t < 0 || t >= nodes) return row;
    const uint64_t *words = tree.mask + ((int64_t)b * tree.tokens + t) * tree.words;
    row.all = true;
    row.lo = words[0];
    if (tree.words > 1) row.hi = words[1];
    return row.cut(nodes);
}

// Length of sequence b and its number of nodes as the kernels see them; what is out of range
// makes the sequence inactive (length 0, no nodes).
__device__ __forceinline__ int checked_tree(const TreeShape &tree, const int32_t *seq_lens, int max_seq_len, int32_t *status,
                                            int b, bool report, int &nodes)
{
    const int len = seq_lens[b];
    nodes = tree.lens ? tree.lens[b] : tree.tokens;
    int flag = 0;
    if (len < 0 || len > max_seq_len) flag = kFlagSeqLenRange;
    else if (len > 0 && (nodes < 0 || nodes > tree.tokens || nodes > len)) flag = kFlagTreeRange;
    if (flag && report && status) atomicOr(status, flag);
    if (flag || len == 0) nodes = 0;
    return flag ? 0 : len;
}

// Row (one token of one head) of a K or V cache that holds a position; 0 where its block cannot be read.
__device__ __forceinline__ int64_t tree_cache_row(const AttnParams &a, int b, int hk, int pos)
{
    if (a.block_table == nullptr) return ((int64_t)b * a.heads + hk) * a.s_max + pos;
    const int phys = a.block_table[(int64_t)b * a.max_blocks_per_seq + pos / a.block_tokens];
    if (phys < 0 || (int64_t)phys >= a.num_phys_blocks) return 0;
    return ((int64_t)phys * a.heads + hk) * a.block_tokens + pos % a.block_tokens;
}

// Whether none of 8 fp16 values is an infinity or a NaN (an exponent field of ones).
__device__ __forceinline__ bool finite8(const uint4 &x)
{
    auto two = [](unsigned w) { return (w & 0x7C00u) != 0x7C00u && (w & 0x7C000000u) != 0x7C000000u; };
    return two(x.x) && two(x.y) && two(x.z) && two(x.w);
}

}  // namespace instinfer
