// C ABI, decode attention over a latent cache: checks, tensor maps and launch.
#include "latent_launch.cuh"
#include "tensor_map.cuh"

namespace {

using namespace instinfer;
using namespace instinfer::api;

int latent_shape(int32_t batch, int32_t q_tokens, int32_t q_heads, int32_t latent_dim, int32_t rope_dim, int32_t max_seq_len)
{
    if (q_tokens <= 0 || q_heads <= 0 || latent_dim <= 0 || rope_dim <= 0 || !sizes_ok(batch, 1, max_seq_len)) return INSTINFER_ERR_INVALID_ARG;
    if (!latent_dims_ok(latent_dim, rope_dim) || q_tokens > kMaxTreeTokens || (int64_t)q_tokens * q_heads > INSTINFER_MAX_LATENT_ROWS)
        return INSTINFER_ERR_UNSUPPORTED;
    return INSTINFER_OK;
}

// Rows of `dims` 16-bit values: a box is 64 of them (128 bytes, the swizzle span) by `box_rows` rows.
bool make_latent_map(CUtensorMap *map, CUtensorMapDataType type, const void *from, int32_t dims, int64_t rows, int64_t batch, int32_t box_rows)
{
    EncodeTiledFn encode = tensor_map_encoder();
    if (encode == nullptr) return false;
    const cuuint64_t row = (cuuint64_t)dims * 2;
    const cuuint64_t size[3] = {(cuuint64_t)dims, (cuuint64_t)rows, (cuuint64_t)batch};
    const cuuint64_t strides[2] = {row, row * (cuuint64_t)rows};
    const cuuint32_t box[3] = {64, (cuuint32_t)box_rows, 1};
    const cuuint32_t elem[3] = {1, 1, 1};
    return encode(map, type, batch > 0 ? 3 : 2, const_cast<void *>(from), size, strides, box, elem, CU_TENSOR_MAP_INTERLEAVE_NONE,
                  CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_128B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

}  // namespace

extern "C" {

int instinfer_decode_attention_latent(void *out, float *lse, const void *q, const void *cache, const int32_t *block_table,
                                      const int32_t *seq_lens, const int32_t *tree_lens, const uint64_t *tree_mask,
                                      int32_t type, int32_t batch, int32_t q_tokens, int32_t q_heads, int32_t latent_dim,
                                      int32_t rope_dim, int32_t s_max, int32_t block_tokens, int32_t max_blocks_per_seq,
                                      int64_t num_phys_blocks, int32_t max_seq_len, float scale, void *workspace,
                                      size_t workspace_bytes, int32_t *status_flags, void *cuda_stream)
{
    const bool paged = block_table != nullptr;
    const int rc = latent_shape(batch, q_tokens, q_heads, latent_dim, rope_dim, max_seq_len);
    if (rc != INSTINFER_OK) return rc;
    if (!std::isfinite(scale)) return INSTINFER_ERR_INVALID_ARG;
    if (type != INSTINFER_F16 && type != INSTINFER_BF16) return INSTINFER_ERR_UNSUPPORTED;
    if (paged) {
        if (block_tokens <= 0 || max_blocks_per_seq <= 0 || num_phys_blocks <= 0 ||
            (int64_t)max_seq_len > (int64_t)max_blocks_per_seq * block_tokens)
            return INSTINFER_ERR_INVALID_ARG;
        if (block_tokens % 8 != 0) return INSTINFER_ERR_UNSUPPORTED;
    } else if (s_max <= 0 || max_seq_len > s_max) {
        return INSTINFER_ERR_INVALID_ARG;
    }
    const int64_t cache_rows = paged ? num_phys_blocks * block_tokens : (int64_t)batch * s_max;
    if (cache_rows >= (int64_t)1 << 31) return INSTINFER_ERR_UNSUPPORTED;
    if (batch == 0) return INSTINFER_OK;
    if (!usable(out) || !usable(q) || !usable(cache) || seq_lens == nullptr || !aligned16(tree_mask)) return INSTINFER_ERR_INVALID_ARG;

    const int64_t rows = (int64_t)q_tokens * q_heads;
    const LatentRows r = latent_rows(rows);
    const LatentCut cut = latent_cut(r, batch, max_seq_len, latent_dim);
    if (!usable(workspace) || workspace_bytes < cut.bytes) return INSTINFER_ERR_WORKSPACE;
    // The merge in whole rows where there are more than 16 warps of 128 dims for every SM.
    const int merge_dims = cut.items * r.block_rows * (latent_dim / 128) > 16 * (int64_t)sm_count() ? latent_dim : 128;
    const int row_parts = (int)ceil_div(r.block_rows, kLatentMergeThreads / 32 / (latent_dim / merge_dims));
    if (cut.items * row_parts >= (int64_t)1 << 31 || cut.most_tiles >= (int64_t)1 << 31 || (int64_t)batch * s_max >= (int64_t)1 << 31)
        return INSTINFER_ERR_INVALID_ARG;

    LatentLaunch t = {};
    LatentParams &p = t.p;
    p.tree.mask = tree_mask;
    p.tree.lens = tree_lens;
    p.tree.tokens = q_tokens;
    p.tree.words = (q_tokens + 63) / 64;
    p.seq_lens = seq_lens;
    p.block_table = block_table;
    p.status = status_flags;
    p.cache = cache;
    p.out = out;
    p.lse = lse;
    unsigned char *start = static_cast<unsigned char *>(workspace);
    p.part_o = static_cast<float *>(workspace);
    p.part_lse = p.part_o + cut.slots * r.block_rows * latent_dim;
    p.item_shares = reinterpret_cast<int2 *>(start + cut.partials_bytes);
    p.num_phys_blocks = paged ? num_phys_blocks : 0;
    p.cache_rows = cache_rows;
    p.batch = batch;
    p.q_heads = q_heads;
    p.rows = (int32_t)rows;
    p.block_rows = r.block_rows;
    p.row_blocks = r.row_blocks;
    p.planes = r.planes;
    p.teams = cut.teams;
    p.tile_shift = cut.tile_shift;
    p.item_cost = cut.item_cost;
    p.max_seq_len = max_seq_len;
    p.s_max = paged ? 0 : s_max;
    p.block_tokens = paged ? block_tokens : 0;
    p.run_tokens = kLatentTile;
    if (paged)
        while (block_tokens % p.run_tokens != 0) p.run_tokens /= 2;      // 64, 32, 16 or 8
    p.max_blocks_per_seq = paged ? max_blocks_per_seq : 0;
    // (the kernels start with a reference of -1e30, unscaled: what scale there is has to tell it from a logit.  Products of
    // 16-bit values that are not huge stay below 1e18, so that this scale and none give the same weights.)
    p.scale = fabsf(scale) < 1e-20f ? copysignf(1e-20f, scale) : scale;
    p.scale_log2e = p.scale * 1.44269504088896340736f;
    const CUtensorMapDataType kind = type == INSTINFER_F16 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16;
    const int32_t dims = latent_dim + rope_dim;
    if (!make_latent_map(&t.map_q, kind, q, dims, rows, batch, r.columns ? r.columns : kPairRows) ||
        !make_latent_map(&t.map_cache, kind, cache, dims, cache_rows, 0, p.run_tokens))
        return INSTINFER_ERR_CUDA;
    t.grid = cut.grid;
    t.merge_grid = (unsigned)(cut.items * row_parts);
    t.row_parts = row_parts;
    t.merge_dims = merge_dims;
    t.stream = static_cast<cudaStream_t>(cuda_stream);
    return type == INSTINFER_F16 ? launch_latent<__half>(r.columns, t) : launch_latent<__nv_bfloat16>(r.columns, t);
}

size_t instinfer_latent_workspace_bytes(int32_t batch, int32_t q_tokens, int32_t q_heads, int32_t latent_dim, int32_t rope_dim,
                                        int32_t max_seq_len)
{
    if (latent_shape(batch, q_tokens, q_heads, latent_dim, rope_dim, max_seq_len) != INSTINFER_OK) return 0;
    if (batch == 0) return 256;
    return latent_cut(latent_rows((int64_t)q_tokens * q_heads), batch, max_seq_len, latent_dim).bytes;
}

}  // extern "C"
