// C ABI, attention of a tree of drafted tokens over the cache: checks, plan and launches.
// Included by instinfer_api.cu after api_grouped.inl, whose planner rules and tensor maps it shares.
#include "tree_launch.cuh"

namespace {

static_assert(kMaxTreeTokens == INSTINFER_MAX_TREE_TOKENS, "limit of the header");

int tree_attention_shape(int32_t batch, int32_t tree_tokens, int32_t q_heads, int32_t kv_heads, int32_t head_dim,
                         int32_t max_seq_len)
{
    if (head_dim <= 0 || tree_tokens <= 0 || q_heads <= 0 || kv_heads <= 0 || q_heads % kv_heads != 0 ||
        !sizes_ok(batch, kv_heads, max_seq_len))
        return INSTINFER_ERR_INVALID_ARG;
    if ((head_dim != 64 && head_dim != 128 && head_dim != 256) || tree_tokens > kMaxTreeTokens ||
        (int64_t)(q_heads / kv_heads) * tree_tokens > INSTINFER_MAX_TREE_ROWS)
        return INSTINFER_ERR_UNSUPPORTED;
    return INSTINFER_OK;
}

// Plan of the warp-level form: the grouped kernel's rules without the search for the best number of chunks (some
// 300 divisions on the host, which every call would pay for the workspace's size).
PlanRules tree_rules(int32_t head_dim)
{
    PlanRules rules = grouped_rules(head_dim);
    rules.block_overhead_tokens = 0;
    return rules;
}

// ---- the tcgen05 form ----

// The grid, and the workspace: partial results (two slots of an item's rows per piece), then the items' pieces and the
// ticket counter.  One function for the size query and the launch, so that they cannot part: the pieces that the kernel
// cuts (TreePieces) are one per block, and where the longest sequences allowed could give every block kTreeDrawnTiles
// tiles, short_pieces more.
struct TreeCut {
    int64_t items, most_tiles;    // tiles (with the items' extra weight) if all sequences were max_seq_len long
    unsigned grid;
    bool draws;
    size_t slot_rows, partials_bytes, ticket_offset, bytes;
};
TreeCut tree_cut(const TreeRows &r, int64_t pairs, int32_t max_seq_len, int32_t head_dim)
{
    TreeCut c;
    c.items = pairs * r.row_blocks;
    c.most_tiles = c.items * (ceil_div(max_seq_len, kTreeTile) + kTreeItemCost);
    c.grid = (unsigned)(c.most_tiles < sm_count() ? c.most_tiles : sm_count());
    c.draws = c.most_tiles >= (int64_t)kTreeDrawnTiles * c.grid;
    const size_t pieces = (size_t)c.grid * (1 + (c.draws ? r.short_pieces : 0)) + 1;
    c.slot_rows = 2 * pieces * r.item_rows;
    c.partials_bytes = (c.slot_rows * (head_dim + 1) * sizeof(float) + 255) / 256 * 256;
    c.ticket_offset = c.partials_bytes + ((size_t)c.items * sizeof(int2) + 255) / 256 * 256;
    c.bytes = c.ticket_offset + 256;
    return c;
}

// Blocks of 16, 32 or 64 tokens, or of a multiple of 128: no tile straddles blocks of another kind.  Head size 64 with at
// most 16 rows is left to the warp-level form: a tile has half the bytes for the same work per token there (16 x 40
// heads x 8k-16k, 16 rows: 450 us, when tcgen05 had an instance for them, against 331 in short runs and 354 sustained;
// 20 rows 473 and 473 against 468 and 559; 32 rows 476 and 483 against 492 and 581; 64 rows 581 and 627 against 937
// and 1077).  The number of tiles does not enter: head size 128, 8 rows, 40 heads, tcgen05 against warp-level: 1
// sequence x 1k 18.1 us against 21.6, x 4k 22.8 against 31.4; 4 x 1k 27.2 against 36.6, x 4k 72.4 against 83.2; 16 x 1k
// 81.9 against 79.6, x 4k 212 against 234; head size 256, 1 x 16 heads x 1k 21.1 against 31.8.
bool tree_umma_shape(int32_t head_dim, int32_t rows, int32_t group, bool paged, int32_t block_tokens)
{
    return group <= kTreeTile && !(head_dim == 64 && rows <= 16) && (!paged || block_tokens == 16 || block_tokens == 32 || block_tokens == 64 || block_tokens % kTreeTile == 0);
}

}  // namespace

extern "C" {

int instinfer_decode_attention_tree(void *out, float *lse, const void *q, const void *k_cache, const void *v_cache,
                                    const int32_t *block_table, const int32_t *seq_lens, const int32_t *tree_lens,
                                    const uint64_t *tree_mask, int32_t batch, int32_t tree_tokens, int32_t q_heads,
                                    int32_t kv_heads, int32_t head_dim, int32_t s_max, int32_t block_tokens,
                                    int32_t max_blocks_per_seq, int64_t num_phys_blocks, int32_t max_seq_len,
                                    float scale, void *workspace, size_t workspace_bytes, int32_t *status_flags,
                                    void *cuda_stream)
{
    const bool paged = block_table != nullptr;
    int rc = tree_attention_shape(batch, tree_tokens, q_heads, kv_heads, head_dim, max_seq_len);
    if (rc != INSTINFER_OK) return rc;
    if (!std::isfinite(scale)) return INSTINFER_ERR_INVALID_ARG;
    if (paged) {
        if (block_tokens <= 0 || max_blocks_per_seq <= 0 || num_phys_blocks <= 0 ||
            (int64_t)max_seq_len > (int64_t)max_blocks_per_seq * block_tokens)
            return INSTINFER_ERR_INVALID_ARG;
        if (block_tokens % kGroupTile != 0) return INSTINFER_ERR_UNSUPPORTED;
    } else if (s_max <= 0 || max_seq_len > s_max) {
        return INSTINFER_ERR_INVALID_ARG;
    }
    if (batch == 0) return INSTINFER_OK;
    if (!usable(out) || !usable(q) || !usable(k_cache) || !usable(v_cache) || !usable(tree_mask) || seq_lens == nullptr)
        return INSTINFER_ERR_INVALID_ARG;

    const int64_t pairs = (int64_t)batch * kv_heads;
    GroupedParams p = {};
    p.group = q_heads / kv_heads;
    p.q_tokens = tree_tokens;
    p.rows = p.group * tree_tokens;
    p.row_groups = (p.rows + kGroupRows - 1) / kGroupRows;
    p.tree.mask = tree_mask;
    p.tree.lens = tree_lens;
    p.tree.tokens = tree_tokens;
    p.tree.words = (tree_tokens + 63) / 64;
    if (!usable(workspace) || workspace_bytes < instinfer_tree_workspace_bytes(batch, tree_tokens, q_heads, kv_heads, head_dim, max_seq_len))
        return INSTINFER_ERR_WORKSPACE;
    const SplitPlan plan = make_plan(pairs * p.row_groups, max_seq_len, tree_rules(head_dim));
    const int64_t grid = pairs * plan.n_splits * p.row_groups;
    if (grid >= (int64_t)1 << 31 || pairs * p.rows >= (int64_t)1 << 31) return INSTINFER_ERR_INVALID_ARG;
    p.a.q = static_cast<const __half *>(q);
    p.a.k = static_cast<const __half *>(k_cache);
    p.a.v = static_cast<const __half *>(v_cache);
    p.a.seq_lens = seq_lens;
    p.a.block_table = block_table;
    p.a.out = static_cast<__half *>(out);
    p.a.lse = lse;
    p.a.status = status_flags;
    p.a.num_phys_blocks = paged ? num_phys_blocks : 0;
    p.a.heads = kv_heads;
    p.a.pairs = (int32_t)pairs;
    p.a.s_max = paged ? 0 : s_max;
    p.a.block_tokens = paged ? block_tokens : 0;
    p.a.max_blocks_per_seq = paged ? max_blocks_per_seq : 0;
    p.a.chunk_tokens = plan.chunk_tokens;
    p.a.n_big = plan.n_big;
    p.a.tail_chunk = plan.tail_chunk;
    p.a.n_splits = plan.n_splits;
    p.a.max_seq_len = max_seq_len;
    p.a.kv_bytes = (paged ? num_phys_blocks * kv_heads * block_tokens : (int64_t)batch * kv_heads * s_max) * head_dim * 2;
    p.a.scale_log2e = scale * 1.44269504088896340736f;
    // (the kernels start with a reference of -1e30, unscaled: what scale there is has to tell it from a logit.
    // Logits of fp16 keys stay below 2^41, so that this scale and none give the same weights.)
    if (fabsf(p.a.scale_log2e) < 1e-20f) p.a.scale_log2e = copysignf(1e-20f, p.a.scale_log2e);
    p.a.part_o = static_cast<float *>(workspace);
    p.a.part_lse = p.a.part_o + (size_t)pairs * plan.n_splits * p.rows * head_dim;
    cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);

    // The tcgen05 form, where the copy engine can take the shape (a cache of 2^31 rows or more, or a
    // driver without the encoder, takes the warp-level one).
    if (g_grouped_path != 1 && tree_umma_shape(head_dim, p.rows, p.group, paged, block_tokens)) {
        const TreeRows rows = tree_rows(tree_tokens, p.group, head_dim);
        const TreeCut cut = tree_cut(rows, pairs, max_seq_len, head_dim);
        const int row_parts = (rows.item_rows + kTreeMergeRows - 1) / kTreeMergeRows;
        const int32_t box = paged && block_tokens < kTreeTile ? block_tokens : kTreeTile;
        TreeLaunch t = {};
        if (cut.items * row_parts < (int64_t)1 << 31 && (int64_t)tree_tokens * q_heads * head_dim < (int64_t)1 << 31 && cut.most_tiles < (int64_t)1 << 31 &&
            make_query_map(&t.map_q, q, batch, tree_tokens, q_heads, p.group, head_dim, rows.nodes_per_block) &&
            make_cache_map(&t.map_k, k_cache, p.a.kv_bytes / (2 * head_dim), head_dim, box) &&
            make_cache_map(&t.map_v, v_cache, p.a.kv_bytes / (2 * head_dim), head_dim, box)) {
            t.p.a = p.a;
            t.p.a.part_lse = p.a.part_o + cut.slot_rows * head_dim;
            t.p.short_pieces = rows.short_pieces;
            unsigned char *start = static_cast<unsigned char *>(workspace);
            t.p.item_pieces = reinterpret_cast<int2 *>(start + cut.partials_bytes);
            t.p.ticket = reinterpret_cast<unsigned *>(start + cut.ticket_offset);
            t.p.tree = p.tree;
            t.p.batch = batch;
            t.p.group = p.group;
            t.p.nodes_per_block = rows.nodes_per_block;
            t.p.row_blocks = rows.row_blocks;
            t.p.item_rows = rows.item_rows;
            t.grid = cut.grid;
            t.merge_grid = (unsigned)(cut.items * row_parts);
            t.row_parts = row_parts;
            t.draws = cut.draws;
            t.stream = stream;
            switch (head_dim) {
            case 64: return paged ? launch_tree<64, true>(rows, t) : launch_tree<64, false>(rows, t);
            case 128: return paged ? launch_tree<128, true>(rows, t) : launch_tree<128, false>(rows, t);
            default: return paged ? launch_tree<256, true>(rows, t) : launch_tree<256, false>(rows, t);
            }
        }
    }
    switch (head_dim) {
    case 64: return paged ? launch_grouped<64, true, true>(p, (unsigned)grid, stream) : launch_grouped<64, false, true>(p, (unsigned)grid, stream);
    case 128: return paged ? launch_grouped<128, true, true>(p, (unsigned)grid, stream) : launch_grouped<128, false, true>(p, (unsigned)grid, stream);
    default: return paged ? launch_grouped<256, true, true>(p, (unsigned)grid, stream) : launch_grouped<256, false, true>(p, (unsigned)grid, stream);
    }
}

size_t instinfer_tree_workspace_bytes(int32_t batch, int32_t tree_tokens, int32_t q_heads, int32_t kv_heads,
                                      int32_t head_dim, int32_t max_seq_len)
{
    if (tree_attention_shape(batch, tree_tokens, q_heads, kv_heads, head_dim, max_seq_len) != INSTINFER_OK) return 0;
    const int64_t pairs = (int64_t)batch * kv_heads;
    if (pairs == 0) return 256;
    const int32_t rows = q_heads / kv_heads * tree_tokens, groups = (rows + kGroupRows - 1) / kGroupRows;
    // enough for either implementation: which one runs also depends on the cache layout
    const size_t warp_level = grouped_workspace_for(pairs, rows, head_dim, make_plan(pairs * groups, max_seq_len, tree_rules(head_dim)));
    const int32_t group = q_heads / kv_heads;
    const size_t umma = group <= kTreeTile ? tree_cut(tree_rows(tree_tokens, group, head_dim), pairs, max_seq_len, head_dim).bytes : 0;
    return warp_level > umma ? warp_level : umma;
}

}  // extern "C"
