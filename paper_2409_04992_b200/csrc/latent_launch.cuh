// How attention over a latent cache is launched: the cut of the rows and of the work, and the entry to the instances,
// which are compiled one type per file (latent_f16.cu, latent_bf16.cu).
#pragma once

#include "api_common.cuh"
#include "latent_kernels.cuh"

namespace instinfer {
namespace api {

// Query rows are cut into row blocks of at most 64, the blocks of a plane take one each.  Up to 8 row blocks all run side
// by side; more are taken four at a time (and rounded up to fours, so that the planes have as much work each).
struct LatentRows {
    int32_t columns;              // 16, 32 or 64: rows of the kernel's instance
    int32_t row_blocks, block_rows, planes;
};
inline LatentRows latent_rows(int64_t rows)
{
    LatentRows r;
    int64_t blocks = ceil_div(rows, 64);
    if (blocks > 8) blocks = ceil_div(blocks, 4) * 4;
    r.row_blocks = (int32_t)blocks;
    r.block_rows = (int32_t)ceil_div(rows, blocks);
    r.row_blocks = (int32_t)ceil_div(rows, r.block_rows);
    r.planes = r.row_blocks <= 8 ? r.row_blocks : 4;
    r.columns = r.block_rows <= 16 ? 16 : r.block_rows <= 32 ? 32 : 64;
    return r;
}

// The grid, and the workspace: partial results (two slots per block), then the items' shares.  One function for the size
// query and the launch.
struct LatentCut {
    int64_t items, most_tiles;    // tiles of a plane (with the items' extra weight) if all sequences were max_seq_len long
    unsigned grid;
    size_t slots, partials_bytes, bytes;
};
inline LatentCut latent_cut(const LatentRows &r, int64_t batch, int32_t max_seq_len, int32_t latent_dim)
{
    LatentCut c;
    c.items = batch * r.row_blocks;
    c.most_tiles = batch * ceil_div(r.row_blocks, r.planes) * (ceil_div(max_seq_len, kLatentTile) + kLatentItemCost);
    const int64_t teams = sm_count() / r.planes;                  // blocks of a plane
    c.grid = (unsigned)((c.most_tiles < teams ? c.most_tiles : teams) * r.planes);
    c.slots = 2 * (size_t)c.grid;
    c.partials_bytes = (c.slots * r.block_rows * (latent_dim + 1) * sizeof(float) + 255) / 256 * 256;
    c.bytes = c.partials_bytes + ((size_t)c.items * sizeof(int2) + 255) / 256 * 256;
    return c;
}

struct LatentLaunch {
    LatentParams p;
    CUtensorMap map_q, map_cache;
    unsigned grid, merge_grid;
    int row_parts;
    cudaStream_t stream;
};

template <typename E>
int launch_latent(int32_t latent_dim, int32_t columns, const LatentLaunch &t);

}  // namespace api
}  // namespace instinfer
