// C ABI, speculative decoding around the attention: ancestor masks, verification of a draft tree,
// keeping the accepted path, and the blocks of a shared paged pool (fork, resize, defragment).
// Included by instinfer_api.cu.
#include "verify_kernels.cuh"

namespace {

static_assert(kMaxLayers == INSTINFER_MAX_LAYERS && kMaxTreeTokens == INSTINFER_MAX_TREE_TOKENS, "limits of the header");

// The layers' cache pointers as a kernel parameter; false if one is unusable.
bool collect_layers(LayerCaches *all, void *const *k, void *const *v, int32_t n_layers)
{
    if (k == nullptr || v == nullptr) return false;
    for (int i = 0; i < n_layers; ++i) {
        if (!usable(k[i]) || !usable(v[i])) return false;
        all->k[i] = static_cast<uint4 *>(k[i]);
        all->v[i] = static_cast<uint4 *>(v[i]);
    }
    return true;
}

// Whether a cache stands at two places of the lists (K and V of one layer are one place): its rows would be moved by different
// blocks, one of which reads what another has moved.
bool listed_twice(const LayerCaches &all, int32_t n_layers)
{
    for (int i = 0; i < n_layers; ++i)
        for (int j = 0; j < i; ++j)
            if (all.k[i] == all.k[j] || all.k[i] == all.v[j] || all.v[i] == all.k[j] || all.v[i] == all.v[j]) return true;
    return false;
}

int launched(cudaError_t err)
{
    return err == cudaSuccess && cudaGetLastError() == cudaSuccess ? INSTINFER_OK : INSTINFER_ERR_CUDA;
}

// Workspace of a resize: the page list's count, the planner's slices, its per-sequence counts, the list.
constexpr size_t kPlanHeaderInts = 64;
size_t resize_ints(int32_t batch) { return kPlanHeaderInts + 3 * (size_t)batch; }
size_t defragment_ints(int64_t blocks) { return kPlanHeaderInts + 2 * (size_t)blocks + 2; }
size_t rounded_bytes(size_t ints) { return (ints * sizeof(int32_t) + 255) / 256 * 256; }

// What the pool entry points share: sizes of the tables and of the pools.
int pool_shape(int32_t batch, int32_t max_blocks_per_seq, int32_t block_tokens, int64_t num_phys_blocks)
{
    if (batch < 0 || max_blocks_per_seq <= 0 || block_tokens <= 0 || num_phys_blocks <= 0) return INSTINFER_ERR_INVALID_ARG;
    if ((int64_t)max_blocks_per_seq * block_tokens > INT32_MAX || num_phys_blocks > INT32_MAX) return INSTINFER_ERR_INVALID_ARG;
    if (block_tokens % 8 != 0 || batch > kMaxPlanBatch || (int64_t)batch * max_blocks_per_seq > (1 << 28)) return INSTINFER_ERR_UNSUPPORTED;
    return INSTINFER_OK;
}

int layers_shape(int32_t n_layers, int32_t heads, int32_t head_dim)
{
    if (n_layers <= 0 || heads <= 0 || head_dim <= 0) return INSTINFER_ERR_INVALID_ARG;
    return n_layers > kMaxLayers || !moved_rows_ok(heads, head_dim) ? INSTINFER_ERR_UNSUPPORTED : INSTINFER_OK;
}

int tree_shape(int32_t batch, int32_t tree_tokens)
{
    if (batch < 0 || batch > 1 << 24 || tree_tokens <= 0) return INSTINFER_ERR_INVALID_ARG;
    return tree_tokens > kMaxTreeTokens ? INSTINFER_ERR_UNSUPPORTED : INSTINFER_OK;
}

template <typename E>
int launch_verify(const VerifyParams &p, int32_t batch, cudaStream_t stream)
{
    // Blocks per sequence: as many as leave every thread at least one 16-byte group of a row.
    const int64_t groups = ceil_div(p.vocab, RowReader<E>::kVec) + 1;       // (a row that starts between boundaries has one more)
    unsigned ctas = 1;
    while (ctas < (unsigned)kVerifyMaxCtas && groups >= (int64_t)ctas * 2 * kVerifyThreads) ctas *= 2;
    // The largest share of a warp, in groups per thread: what the instances hold, 32 elements at most (16 of 64 bits
    // and 16 of 32 would leave room for more threads, but a second wave costs less than a second pass over memory).
    constexpr int kVec = RowReader<E>::kVec;
    const int64_t held = ceil_div(ceil_div(groups, (int64_t)ctas * kVerifyWarps), 32);
    if (held <= 8 / kVec) return launched(launch_clustered(verify_tree_kernel<E, 8 / kVec, 256>, (unsigned)batch * ctas, ctas, 256, 0, stream, p));
    if (held <= 16 / kVec) return launched(launch_clustered(verify_tree_kernel<E, 16 / kVec, 256>, (unsigned)batch * ctas, ctas, 256, 0, stream, p));
    if (held <= 32 / kVec) return launched(launch_clustered(verify_tree_kernel<E, 32 / kVec, 256>, (unsigned)batch * ctas, ctas, 256, 0, stream, p));
    if (held <= 64 / kVec) return launched(launch_clustered(verify_tree_kernel<E, 32 / kVec, 512>, (unsigned)batch * ctas, ctas, 512, 0, stream, p));
    return launched(launch_clustered(verify_tree_streamed_kernel<E>, (unsigned)batch * ctas, ctas, kVerifyThreads, 0, stream, p));
}

// Moving pages is bound by HBM: enough blocks to fill the GPU, fewer where the list cannot be long.
unsigned move_grid(int64_t most_pages, int32_t n_layers, int64_t page_segs)
{
    const int64_t pieces = most_pages * n_layers * 2 * ceil_div(page_segs, kMoveSegs);
    const int64_t full = (int64_t)sm_count() * 8;
    return (unsigned)(pieces < 1 ? 1 : pieces < full ? pieces : full);
}

}  // namespace

extern "C" {

int instinfer_tree_mask(uint64_t *tree_mask, const int32_t *parents, const int32_t *tree_lens, int32_t batch,
                        int32_t tree_tokens, int32_t *status_flags, void *cuda_stream)
{
    const int rc = tree_shape(batch, tree_tokens);
    if (rc != INSTINFER_OK) return rc;
    if (batch == 0) return INSTINFER_OK;
    if (!usable(tree_mask) || parents == nullptr) return INSTINFER_ERR_INVALID_ARG;
    const int32_t words = (tree_tokens + 63) / 64;
    return launched(launch_overlapped(tree_mask_kernel, (unsigned)batch, kMaxTreeTokens, 0, static_cast<cudaStream_t>(cuda_stream),
                                      tree_mask, parents, tree_lens, tree_tokens, words, status_flags));
}

int instinfer_verify_tree(int32_t *path, int32_t *path_lens, int32_t *out_tokens, const void *target_probs,
                          const void *draft_probs, int32_t probs_type, int64_t row_stride, const int32_t *tokens,
                          const int32_t *parents, const int32_t *tree_lens, const float *uniforms, int32_t batch,
                          int32_t tree_tokens, int32_t vocab, int32_t *status_flags, void *cuda_stream)
{
    const int rc = tree_shape(batch, tree_tokens);
    if (rc != INSTINFER_OK) return rc;
    if (vocab <= 0 || vocab > 1 << 30 || row_stride < vocab) return INSTINFER_ERR_INVALID_ARG;
    if (probs_type != INSTINFER_F32 && probs_type != INSTINFER_F16 && probs_type != INSTINFER_BF16) return INSTINFER_ERR_UNSUPPORTED;
    if (batch == 0) return INSTINFER_OK;
    if (path == nullptr || path_lens == nullptr || out_tokens == nullptr || !usable(target_probs) ||
        !aligned16(draft_probs) || tokens == nullptr || parents == nullptr || uniforms == nullptr)
        return INSTINFER_ERR_INVALID_ARG;
    VerifyParams p = {};
    p.path = path;
    p.path_lens = path_lens;
    p.out_tokens = out_tokens;
    p.target = target_probs;
    p.draft = draft_probs;
    p.tokens = tokens;
    p.parents = parents;
    p.tree_lens = tree_lens;
    p.uniforms = uniforms;
    p.status = status_flags;
    p.row_stride = row_stride;
    p.tree_tokens = tree_tokens;
    p.vocab = vocab;
    cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    return probs_type == INSTINFER_F32 ? launch_verify<float>(p, batch, stream)
           : probs_type == INSTINFER_F16 ? launch_verify<__half>(p, batch, stream)
                                         : launch_verify<__nv_bfloat16>(p, batch, stream);
}

int instinfer_kv_keep_path(void *const *k_caches, void *const *v_caches, int32_t n_layers, const int32_t *path,
                           const int32_t *path_lens, const int32_t *tree_lens, const int32_t *seq_lens,
                           int32_t *new_lens, const int32_t *block_table, int32_t max_blocks_per_seq,
                           int32_t block_tokens, int64_t num_phys_blocks, int32_t batch, int32_t tree_tokens,
                           int32_t heads, int32_t head_dim, int32_t s_max, int32_t *status_flags, void *cuda_stream)
{
    int rc = tree_shape(batch, tree_tokens);
    if (rc == INSTINFER_OK) rc = layers_shape(n_layers, heads, head_dim);
    if (rc != INSTINFER_OK) return rc;
    if (block_table) {
        if (max_blocks_per_seq <= 0 || block_tokens <= 0 || num_phys_blocks <= 0) return INSTINFER_ERR_INVALID_ARG;
        if (block_tokens % 8 != 0) return INSTINFER_ERR_UNSUPPORTED;
    } else if (s_max <= 0) {
        return INSTINFER_ERR_INVALID_ARG;
    }
    if (batch == 0) return INSTINFER_OK;
    LayerCaches caches = {};
    if (path == nullptr || path_lens == nullptr || seq_lens == nullptr || new_lens == nullptr || new_lens == seq_lens ||
        !collect_layers(&caches, k_caches, v_caches, n_layers))
        return INSTINFER_ERR_INVALID_ARG;
    // (layers of K and V caches are no pairs of one cache; latent ones may be, so that their lists are looked at)
    if (!append_head_dim_ok(head_dim) && listed_twice(caches, n_layers)) return INSTINFER_ERR_INVALID_ARG;
    KeepPathParams p = {};
    p.path = path;
    p.path_lens = path_lens;
    p.tree_lens = tree_lens;
    p.seq_lens = seq_lens;
    p.new_lens = new_lens;
    p.block_table = block_table;
    p.status = status_flags;
    p.num_phys_blocks = num_phys_blocks;
    p.batch = batch;
    p.tree_tokens = tree_tokens;
    p.heads = heads;
    p.s_max = s_max;
    p.block_tokens = block_tokens;
    p.max_blocks_per_seq = max_blocks_per_seq;
    p.segs_per_row = head_dim / 8;
    const int64_t column_blocks = ceil_div((int64_t)heads * p.segs_per_row, kKeepThreads);
    const int64_t grid = column_blocks * batch * n_layers;
    if (grid >= (int64_t)1 << 31) return INSTINFER_ERR_INVALID_ARG;
    p.column_blocks = (int32_t)column_blocks;
    p.cache_rows = block_table ? num_phys_blocks * heads * block_tokens : (int64_t)batch * heads * s_max;
    return launched(launch_overlapped(kv_keep_path_kernel, (unsigned)grid, kKeepThreads, 0,
                                      static_cast<cudaStream_t>(cuda_stream), p, caches));
}

int instinfer_kv_fork(int32_t *block_table, int32_t *block_refs, int32_t *seq_lens, const int32_t *src,
                      const int32_t *dst, int32_t n_forks, int32_t max_blocks_per_seq, int32_t block_tokens,
                      int64_t num_phys_blocks, int32_t batch, int32_t *status_flags, void *cuda_stream)
{
    const int rc = pool_shape(batch, max_blocks_per_seq, block_tokens, num_phys_blocks);
    if (rc != INSTINFER_OK) return rc;
    if (n_forks < 0 || n_forks > batch) return INSTINFER_ERR_INVALID_ARG;
    if (n_forks == 0) return INSTINFER_OK;
    if (block_table == nullptr || block_refs == nullptr || seq_lens == nullptr || src == nullptr || dst == nullptr)
        return INSTINFER_ERR_INVALID_ARG;
    ForkParams p = {};
    p.block_table = block_table;
    p.block_refs = block_refs;
    p.seq_lens = seq_lens;
    p.src = src;
    p.dst = dst;
    p.status = status_flags;
    p.num_phys_blocks = num_phys_blocks;
    p.n_forks = n_forks;
    p.batch = batch;
    p.block_tokens = block_tokens;
    p.max_blocks_per_seq = max_blocks_per_seq;
    return launched(launch_overlapped(kv_fork_kernel, (unsigned)n_forks, kForkThreads, 0, static_cast<cudaStream_t>(cuda_stream), p));
}

size_t instinfer_kv_resize_workspace_bytes(int32_t batch, int64_t num_phys_blocks)
{
    if (batch < 0 || batch > kMaxPlanBatch || num_phys_blocks <= 0 || num_phys_blocks > INT32_MAX) return 0;
    return rounded_bytes(resize_ints(batch));
}

int instinfer_kv_resize(void *const *k_pools, void *const *v_pools, int32_t n_layers, int32_t *block_table,
                        int32_t *block_refs, const int32_t *seq_lens, const int32_t *want_lens, int32_t *new_lens,
                        int32_t max_blocks_per_seq, int32_t block_tokens, int64_t num_phys_blocks, int32_t batch,
                        int32_t heads, int32_t head_dim, void *workspace, size_t workspace_bytes,
                        int32_t *status_flags, void *cuda_stream)
{
    int rc = pool_shape(batch, max_blocks_per_seq, block_tokens, num_phys_blocks);
    if (rc == INSTINFER_OK) rc = layers_shape(n_layers, heads, head_dim);
    if (rc != INSTINFER_OK) return rc;
    if (batch == 0) return INSTINFER_OK;
    LayerCaches caches = {};
    if (block_table == nullptr || block_refs == nullptr || seq_lens == nullptr || want_lens == nullptr || new_lens == nullptr ||
        !collect_layers(&caches, k_pools, v_pools, n_layers))
        return INSTINFER_ERR_INVALID_ARG;
    if (!usable(workspace) || workspace_bytes < rounded_bytes(resize_ints(batch))) return INSTINFER_ERR_WORKSPACE;
    int32_t *ws = static_cast<int32_t *>(workspace);
    ResizeParams p = {};
    p.block_table = block_table;
    p.block_refs = block_refs;
    p.seq_lens = seq_lens;
    p.want_lens = want_lens;
    p.new_lens = new_lens;
    p.status = status_flags;
    p.num_phys_blocks = num_phys_blocks;
    p.batch = batch;
    p.block_tokens = block_tokens;
    p.max_blocks_per_seq = max_blocks_per_seq;
    p.list.count = ws;
    p.slices = ws + 1;
    p.counts = ws + kPlanHeaderInts;
    p.list.pages = p.counts + batch;
    const size_t smem = (size_t)batch * 4 * sizeof(int32_t);
    if (smem > 48 * 1024) {
        static bool done[kMaxDevices] = {};
        int dev = 0;
        if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= kMaxDevices) return INSTINFER_ERR_CUDA;
        if (!done[dev]) {
            if (cudaFuncSetAttribute(kv_resize_plan_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                     kMaxPlanBatch * 4 * (int)sizeof(int32_t)) != cudaSuccess) {
                (void)cudaGetLastError();
                return INSTINFER_ERR_CUDA;
            }
            done[dev] = true;
        }
    }
    cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    rc = launched(launch_clustered(kv_resize_plan_kernel, kPlanCtas, kPlanCtas, kPlanThreads, smem, stream, p));
    if (rc != INSTINFER_OK) return rc;
    const int64_t page_segs = (int64_t)heads * block_tokens * head_dim / 8;
    return launched(launch_overlapped(kv_move_pages_kernel<false>, move_grid(batch, n_layers, page_segs), kMoveThreads, 0, stream,
                                      p.list, n_layers, page_segs, num_phys_blocks, status_flags, DefragmentParams{}, caches));
}

size_t instinfer_kv_defragment_workspace_bytes(int64_t num_phys_blocks)
{
    if (num_phys_blocks <= 0 || num_phys_blocks > INT32_MAX) return 0;
    return rounded_bytes(defragment_ints(num_phys_blocks));
}

int instinfer_kv_defragment(void *const *k_pools, void *const *v_pools, int32_t n_layers, const int32_t *block_table,
                            int32_t *new_block_table, const int32_t *block_refs, int32_t *new_block_refs,
                            const int32_t *seq_lens, int32_t *blocks_used, int32_t max_blocks_per_seq,
                            int32_t block_tokens, int64_t num_phys_blocks, int32_t batch, int32_t heads,
                            int32_t head_dim, void *workspace, size_t workspace_bytes, int32_t *status_flags,
                            void *cuda_stream)
{
    int rc = pool_shape(batch, max_blocks_per_seq, block_tokens, num_phys_blocks);
    if (rc == INSTINFER_OK) rc = layers_shape(n_layers, heads, head_dim);
    if (rc != INSTINFER_OK) return rc;
    if (batch == 0) return INSTINFER_OK;
    LayerCaches caches = {};
    if (block_table == nullptr || new_block_table == nullptr || block_refs == nullptr || new_block_refs == nullptr ||
        seq_lens == nullptr || blocks_used == nullptr || !collect_layers(&caches, k_pools, v_pools, n_layers))
        return INSTINFER_ERR_INVALID_ARG;
    if (!usable(workspace) || workspace_bytes < rounded_bytes(defragment_ints(num_phys_blocks))) return INSTINFER_ERR_WORKSPACE;
    int32_t *ws = static_cast<int32_t *>(workspace);
    DefragmentParams p = {};
    p.block_table = block_table;
    p.new_table = new_block_table;
    p.block_refs = block_refs;
    p.new_refs = new_block_refs;
    p.seq_lens = seq_lens;
    p.blocks_used = blocks_used;
    p.status = status_flags;
    p.num_phys_blocks = num_phys_blocks;
    p.batch = batch;
    p.block_tokens = block_tokens;
    p.max_blocks_per_seq = max_blocks_per_seq;
    p.list.count = ws;
    p.slices = ws + 1;
    p.map = ws + kPlanHeaderInts;
    p.list.pages = p.map + num_phys_blocks;
    cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    rc = launched(launch_clustered(kv_defragment_plan_kernel, kPlanCtas, kPlanCtas, kPlanThreads, 0, stream, p));
    if (rc != INSTINFER_OK) return rc;
    const int64_t page_segs = (int64_t)heads * block_tokens * head_dim / 8;
    return launched(launch_overlapped(kv_move_pages_kernel<true>, move_grid(num_phys_blocks / 2 + 1, n_layers, page_segs), kMoveThreads,
                                      0, stream, p.list, n_layers, page_segs, num_phys_blocks, status_flags, p, caches));
}

}  // extern "C"
