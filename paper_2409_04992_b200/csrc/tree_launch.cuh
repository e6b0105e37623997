// How a draft tree's attention is launched on the tcgen05 kernels: the cut of the rows, and the entry to the
// instances, which are compiled one head size per file (tree_d64.cu, tree_d128.cu, tree_d256.cu).
#pragma once

#include "api_common.cuh"
#include "tree_umma_common.cuh"

namespace instinfer {
namespace api {

// How the rows of a (sequence, KV head) are cut.  Up to 64 rows: one block for the kernel with the tokens as
// the long side (N columns).  More: row blocks of at most 128 rows, whole nodes each; with more than one,
// two share every K and V tile (head size 256 has no room in tensor memory for two).
struct TreeRows {
    int32_t columns;              // 16, 32 or 64; 0: the kernel with the rows as the long side
    int32_t streams, nodes_per_block, row_blocks, item_rows;
    int32_t short_pieces;         // drawn pieces per block: fewer where a partial result is larger
};
inline TreeRows tree_rows(int32_t tree_tokens, int32_t group, int32_t head_dim)
{
    TreeRows r;
    const int32_t rows = tree_tokens * group;
    r.columns = rows <= 16 ? 16 : rows <= 32 ? 32 : rows <= 64 ? 64 : 0;
    const int32_t most = kTreeTile / group;
    const int32_t blocks = r.columns ? 1 : (tree_tokens + most - 1) / most;
    r.streams = blocks > 1 && head_dim != 256 ? 2 : 1;
    r.row_blocks = (blocks + r.streams - 1) / r.streams;
    r.nodes_per_block = (tree_tokens + r.row_blocks * r.streams - 1) / (r.row_blocks * r.streams);
    r.item_rows = r.streams * r.nodes_per_block * group;
    r.short_pieces = r.columns ? 4 : 2;
    return r;
}

struct TreeLaunch {
    TreeParams p;
    CUtensorMap map_q, map_k, map_v;
    unsigned grid, merge_grid;
    int row_parts;
    bool draws;                   // there may be enough tiles for drawn pieces
    cudaStream_t stream;
};

// The kernel for the rows' cut, and the merge behind it.
template <int D, bool kPaged>
int launch_tree(const TreeRows &rows, const TreeLaunch &t);

}  // namespace api
}  // namespace instinfer
