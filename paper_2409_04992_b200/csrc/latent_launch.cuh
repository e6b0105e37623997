// How attention over a latent cache is launched: the cut of the rows and of the work, and the entry to the instances,
// which are compiled one type per file (latent_f16.cu, latent_bf16.cu).
#pragma once

#include "api_common.cuh"
#include "latent_pair_kernels.cuh"

namespace instinfer {
namespace api {

// Up to 32 rows: one row block for the kernel with the tokens as the long side (`columns` of the instance).  More: row blocks of at most
// 128 rows for pairs of SMs.  Up to 4 row blocks all run side by side (a plane each); more are taken two at a time.
struct LatentRows {
    int32_t columns;              // 16, 32; 0: pairs
    int32_t row_blocks, block_rows, planes;
};
inline LatentRows latent_rows(int64_t rows)
{
    LatentRows r;
    r.columns = rows <= 16 ? 16 : rows <= 32 ? 32 : 0;
    int64_t blocks = r.columns ? 1 : ceil_div(rows, 2 * kPairRows);
    if (blocks > 4) blocks = ceil_div(blocks, 2) * 2;
    r.block_rows = (int32_t)ceil_div(rows, blocks);
    r.row_blocks = (int32_t)ceil_div(rows, r.block_rows);
    r.planes = r.row_blocks <= 4 ? r.row_blocks : 2;
    return r;
}

// The grid, and the workspace: partial results (two slots per block or pair of blocks), then the items' shares.  One
// function for the size query and the launch.
struct LatentCut {
    int32_t tile_shift, item_cost;
    int64_t items, most_tiles;    // tiles of a plane (with the items' extra weight) if all sequences were max_seq_len long
    int32_t teams;                // blocks (or pairs) of a plane
    unsigned grid;
    size_t slots, partials_bytes, bytes;
};
inline LatentCut latent_cut(const LatentRows &r, int64_t batch, int32_t max_seq_len, int32_t latent_dim)
{
    LatentCut c;
    c.tile_shift = r.columns ? 6 : 7;
    c.item_cost = r.columns ? 3 : 2;
    c.items = batch * r.row_blocks;
    c.most_tiles = batch * ceil_div(r.row_blocks, r.planes) * (ceil_div(max_seq_len, (int64_t)1 << c.tile_shift) + c.item_cost);
    const int64_t teams = sm_count() / (r.columns ? 1 : 2) / r.planes;
    c.teams = (int32_t)(c.most_tiles < teams ? c.most_tiles : teams);
    c.grid = (unsigned)(c.teams * r.planes * (r.columns ? 1 : 2));
    c.slots = 2 * (size_t)c.teams * r.planes;
    c.partials_bytes = (c.slots * r.block_rows * (latent_dim + 1) * sizeof(float) + 255) / 256 * 256;
    c.bytes = c.partials_bytes + ((size_t)c.items * sizeof(int2) + 255) / 256 * 256;
    return c;
}

struct LatentLaunch {
    LatentParams p;
    CUtensorMap map_q, map_cache;
    unsigned grid, merge_grid;
    int row_parts, merge_dims;    // blocks of an item, dims of a warp of the merge
    cudaStream_t stream;
};

template <typename E>
int launch_latent(int32_t columns, const LatentLaunch &t);

}  // namespace api
}  // namespace instinfer
