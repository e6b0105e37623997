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
    int32_t short_pieces;         // drawn pieces per block: fewer where a partial result is larger
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
    r.short_pieces = r.columns == 16 ? 4 : 2;
    return r;
}

// The grid, and the workspace: partial results (two slots per piece that a plane can be cut into), then the items' pieces
// and the ticket counters.  One function for the size query and the launch.
struct LatentCut {
    int64_t items, most_tiles;    // tiles of a plane (with the items' extra weight) if all sequences were max_seq_len long
    unsigned teams;               // blocks of a plane
    bool draws;
    int64_t plane_slots;
    size_t slots, partials_bytes, ticket_offset, bytes;
};
inline LatentCut latent_cut(const LatentRows &r, int64_t batch, int32_t max_seq_len, int32_t latent_dim)
{
    LatentCut c;
    c.items = batch * r.row_blocks;
    c.most_tiles = batch * ceil_div(r.row_blocks, r.planes) * (ceil_div(max_seq_len, kLatentTile) + kLatentItemCost);
    const int64_t blocks = sm_count() / r.planes;
    c.teams = (unsigned)(c.most_tiles < blocks ? c.most_tiles : blocks);
    c.draws = c.most_tiles >= (int64_t)kTreeDrawnTiles * c.teams;
    c.plane_slots = 2 * ((int64_t)c.teams * (1 + (c.draws ? r.short_pieces : 0)) + 1);
    c.slots = (size_t)c.plane_slots * r.planes;
    c.partials_bytes = (c.slots * r.block_rows * (latent_dim + 1) * sizeof(float) + 255) / 256 * 256;
    c.ticket_offset = c.partials_bytes + ((size_t)c.items * sizeof(int2) + 255) / 256 * 256;
    c.bytes = c.ticket_offset + 256;
    return c;
}

struct LatentLaunch {
    LatentParams p;
    CUtensorMap map_q, map_cache;
    unsigned grid, merge_grid;
    int row_parts;
    bool draws;                   // there may be enough tiles for drawn pieces
    cudaStream_t stream;
};

template <typename E>
int launch_latent(int32_t latent_dim, int32_t columns, const LatentLaunch &t);

}  // namespace api
}  // namespace instinfer
