// C ABI, rotary positions: the pairs' frequencies (host), and the appends that turn queries and keys on the way.
#include "api_common.cuh"

#include <type_traits>

#include "rope_kernels.cuh"

namespace {

using namespace instinfer;
using namespace instinfer::api;

constexpr double kPi = 3.14159265358979323846;

// What the two appends check alike, and the sizes that follow from it.
int append_shape(int32_t batch, int32_t max_new, const int32_t *block_table, int32_t max_blocks_per_seq, int32_t block_tokens,
                 int64_t num_phys_blocks, int32_t s_max)
{
    if (batch < 0 || max_new < 0 || batch > 1 << 24) return INSTINFER_ERR_INVALID_ARG;
    if (block_table != nullptr) {
        if (max_blocks_per_seq <= 0 || block_tokens <= 0 || num_phys_blocks <= 0) return INSTINFER_ERR_INVALID_ARG;
        if (block_tokens % 8 != 0) return INSTINFER_ERR_UNSUPPORTED;
    } else if (s_max <= 0) {
        return INSTINFER_ERR_INVALID_ARG;
    }
    return INSTINFER_OK;
}

// Strides are in elements; every token and head starts on a 16-byte boundary.
bool stride_ok(int64_t stride, int64_t least, int32_t element_bytes)
{
    return stride >= least && stride < (int64_t)1 << 40 && stride * element_bytes % 16 == 0;
}

// Parts of `dims` values, of tokens q_stride and of heads q_head_stride apart, do not overlap: a token's heads lie before the next
// token's, or a head's tokens before the next head's.
bool parts_apart(int64_t q_stride, int64_t q_head_stride, int64_t tokens, int64_t heads, int64_t dims)
{
    return heads - 1 <= (q_stride - dims) / q_head_stride || tokens - 1 <= (q_head_stride - dims) / q_stride;
}

bool frequencies_ok(const double *frequencies) { return frequencies != nullptr && (reinterpret_cast<uintptr_t>(frequencies) & 7u) == 0; }

template <typename In, typename Out, bool kLatent>
int launch_rope(RopeParams p, bool interleaved, cudaStream_t stream)
{
    // Many tokens: four a block, whose sines keep all its threads busy once.  Few: the blocks of a token share its units
    // until every SM has two blocks or a thread has one unit.
    const int64_t tokens = (int64_t)p.batch * p.max_new;
    const int64_t units = (int64_t)(p.q_heads + p.kv_heads) * p.head_units + (kLatent ? 1 : p.kv_heads) * (int64_t)p.v_units;
    const int64_t wide = ceil_div(units, kRopeThreads), wanted = 2 * (int64_t)sm_count();
    p.tokens_per_block = tokens >= 4 * kRopeTokens * (int64_t)sm_count() ? kRopeTokens : 1;
    const int64_t parts = ceil_div(wanted, tokens);
    p.parts = (int32_t)(p.tokens_per_block > 1 ? 1 : parts < wide ? parts : wide);
    const int64_t grid = ceil_div(tokens, p.tokens_per_block) * p.parts;
    if (grid >= (int64_t)1 << 31 || units >= 1 << 30) return INSTINFER_ERR_INVALID_ARG;
    const cudaError_t err = interleaved
        ? launch_overlapped(rope_append_kernel<In, Out, true, kLatent>, (unsigned)grid, kRopeThreads, 0, stream, p)
        : launch_overlapped(rope_append_kernel<In, Out, false, kLatent>, (unsigned)grid, kRopeThreads, 0, stream, p);
    return err == cudaSuccess && cudaGetLastError() == cudaSuccess ? INSTINFER_OK : INSTINFER_ERR_CUDA;
}

}  // namespace

extern "C" {

int instinfer_rope_frequencies(double *frequencies, float *magnitude, int32_t rope_dim, double base, int32_t scaling,
                               double factor, int32_t trained_len, double slow_turns, double fast_turns)
{
    if (frequencies == nullptr || magnitude == nullptr || rope_dim <= 0 || rope_dim % 2 != 0 || !(base > 0) || !std::isfinite(base))
        return INSTINFER_ERR_INVALID_ARG;
    if (scaling != INSTINFER_ROPE_PLAIN && scaling != INSTINFER_ROPE_LINEAR && scaling != INSTINFER_ROPE_BY_PARTS) return INSTINFER_ERR_UNSUPPORTED;
    if (scaling != INSTINFER_ROPE_PLAIN && (!(factor >= 1) || !std::isfinite(factor))) return INSTINFER_ERR_INVALID_ARG;
    if (scaling == INSTINFER_ROPE_BY_PARTS &&
        (trained_len <= 0 || !(slow_turns >= 0) || !(fast_turns > slow_turns) || !std::isfinite(fast_turns)))
        return INSTINFER_ERR_INVALID_ARG;
    *magnitude = 1.f;
    for (int i = 0; i < rope_dim / 2; ++i) {
        const double plain = std::pow(base, -2.0 * i / rope_dim);
        double kept = 1.0;                        // of the plain frequency; the rest is divided by the factor
        if (scaling == INSTINFER_ROPE_LINEAR) {
            kept = 0.0;
        } else if (scaling == INSTINFER_ROPE_BY_PARTS) {
            kept = (trained_len * plain / (2 * kPi) - slow_turns) / (fast_turns - slow_turns);
            kept = kept < 0 ? 0 : kept > 1 ? 1 : kept;
        }
        frequencies[i] = scaling == INSTINFER_ROPE_PLAIN ? plain : kept * plain + (1 - kept) * plain / factor;
    }
    if (scaling == INSTINFER_ROPE_BY_PARTS) *magnitude = (float)(0.1 * std::log(factor) + 1.0);
    return INSTINFER_OK;
}

int instinfer_rope_append(void *q_out, void *k_cache, void *v_cache, const void *q, const void *k_new, const void *v_new,
                          int32_t type, int64_t q_stride, int64_t k_stride, int64_t v_stride, const double *frequencies,
                          int32_t rope_dim, int32_t interleaved, float magnitude, const int32_t *positions,
                          const int32_t *seq_lens, const int32_t *new_lens, const int32_t *block_table,
                          int32_t max_blocks_per_seq, int32_t block_tokens, int64_t num_phys_blocks, int32_t batch,
                          int32_t max_new, int32_t q_heads, int32_t kv_heads, int32_t head_dim, int32_t s_max,
                          int32_t *status_flags, void *cuda_stream)
{
    if (q_heads < 0 || kv_heads <= 0 || head_dim <= 0 || rope_dim <= 0 || rope_dim > head_dim || !std::isfinite(magnitude))
        return INSTINFER_ERR_INVALID_ARG;
    int rc = append_shape(batch, max_new, block_table, max_blocks_per_seq, block_tokens, num_phys_blocks, s_max);
    if (rc != INSTINFER_OK) return rc;
    if (!append_head_dim_ok(head_dim) || rope_dim % 16 != 0) return INSTINFER_ERR_UNSUPPORTED;
    if (type != INSTINFER_F32 && type != INSTINFER_F16 && type != INSTINFER_BF16) return INSTINFER_ERR_UNSUPPORTED;
    if ((int64_t)batch * kv_heads > (int64_t)1 << 24 || q_heads > 1 << 20) return INSTINFER_ERR_INVALID_ARG;
    const int32_t bytes = type == INSTINFER_F32 ? 4 : 2;
    if ((q_heads > 0 && !stride_ok(q_stride, (int64_t)q_heads * head_dim, bytes)) || !stride_ok(k_stride, (int64_t)kv_heads * head_dim, bytes) ||
        !stride_ok(v_stride, (int64_t)kv_heads * head_dim, bytes))
        return INSTINFER_ERR_INVALID_ARG;
    if (batch == 0 || max_new == 0) return INSTINFER_OK;
    if (!usable(k_cache) || !usable(v_cache) || !usable(k_new) || !usable(v_new) || !frequencies_ok(frequencies) || seq_lens == nullptr ||
        (q_heads > 0 && (!usable(q) || !usable(q_out))))
        return INSTINFER_ERR_INVALID_ARG;
    RopeParams p = {};
    p.q = q;
    p.k = k_new;
    p.v = v_new;
    p.q_out = q_out;
    p.k_cache = k_cache;
    p.v_cache = v_cache;
    p.frequencies = frequencies;
    p.positions = positions;
    p.seq_lens = seq_lens;
    p.new_lens = new_lens;
    p.block_table = block_table;
    p.status = status_flags;
    p.q_stride = q_stride;
    p.k_stride = k_stride;
    p.v_stride = v_stride;
    p.q_head_stride = head_dim;
    p.q_out_stride = (int64_t)q_heads * head_dim;
    p.q_out_head_stride = head_dim;
    p.num_phys_blocks = num_phys_blocks;
    p.cache_rows = block_table ? num_phys_blocks * kv_heads * block_tokens : (int64_t)batch * kv_heads * s_max;
    p.batch = batch;
    p.max_new = max_new;
    p.q_heads = q_heads;
    p.kv_heads = kv_heads;
    p.head_units = p.v_units = head_dim / 16;
    p.pairs = rope_dim / 2;
    p.s_max = s_max;
    p.block_tokens = block_tokens;
    p.max_blocks_per_seq = max_blocks_per_seq;
    p.magnitude = magnitude;
    cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    return type == INSTINFER_F32 ? launch_rope<float, __half, false>(p, interleaved != 0, stream)
           : type == INSTINFER_F16 ? launch_rope<__half, __half, false>(p, interleaved != 0, stream)
                                   : launch_rope<__nv_bfloat16, __half, false>(p, interleaved != 0, stream);
}

int instinfer_latent_append(void *q_out, void *cache, const void *q_rope, const void *latent_new, const void *rope_new,
                            int32_t type, int64_t q_stride, int64_t q_head_stride, int64_t latent_stride, int64_t rope_stride,
                            const double *frequencies, int32_t interleaved, float magnitude, const int32_t *positions,
                            const int32_t *seq_lens, const int32_t *new_lens, const int32_t *block_table,
                            int32_t max_blocks_per_seq, int32_t block_tokens, int64_t num_phys_blocks, int32_t batch,
                            int32_t max_new, int32_t q_heads, int32_t latent_dim, int32_t rope_dim, int32_t s_max,
                            int32_t *status_flags, void *cuda_stream)
{
    if (q_heads < 0 || latent_dim <= 0 || rope_dim <= 0 || !std::isfinite(magnitude)) return INSTINFER_ERR_INVALID_ARG;
    int rc = append_shape(batch, max_new, block_table, max_blocks_per_seq, block_tokens, num_phys_blocks, s_max);
    if (rc != INSTINFER_OK) return rc;
    if (!latent_dims_ok(latent_dim, rope_dim) || (type != INSTINFER_F16 && type != INSTINFER_BF16)) return INSTINFER_ERR_UNSUPPORTED;
    if (q_heads > 1 << 20) return INSTINFER_ERR_INVALID_ARG;
    if ((q_heads > 0 && (!stride_ok(q_head_stride, rope_dim, 2) || !stride_ok(q_stride, rope_dim, 2) ||
                         !parts_apart(q_stride, q_head_stride, (int64_t)batch * max_new, q_heads, rope_dim))) ||
        !stride_ok(latent_stride, latent_dim, 2) || !stride_ok(rope_stride, rope_dim, 2))
        return INSTINFER_ERR_INVALID_ARG;
    if (batch == 0 || max_new == 0) return INSTINFER_OK;
    if (!usable(cache) || !usable(latent_new) || !usable(rope_new) || !frequencies_ok(frequencies) || seq_lens == nullptr ||
        (q_heads > 0 && (!usable(q_rope) || !usable(q_out))))
        return INSTINFER_ERR_INVALID_ARG;
    RopeParams p = {};
    p.q = q_rope;
    p.k = rope_new;
    p.v = latent_new;
    p.q_out = q_heads > 0 ? static_cast<char *>(q_out) + 2 * latent_dim : nullptr;
    p.k_cache = cache;
    p.frequencies = frequencies;
    p.positions = positions;
    p.seq_lens = seq_lens;
    p.new_lens = new_lens;
    p.block_table = block_table;
    p.status = status_flags;
    p.q_stride = q_stride;
    p.k_stride = rope_stride;
    p.v_stride = latent_stride;
    p.q_head_stride = q_head_stride;
    p.q_out_head_stride = latent_dim + rope_dim;
    p.q_out_stride = q_heads * p.q_out_head_stride;
    p.num_phys_blocks = num_phys_blocks;
    p.cache_rows = block_table ? num_phys_blocks * block_tokens : (int64_t)batch * s_max;
    p.batch = batch;
    p.max_new = max_new;
    p.q_heads = q_heads;
    p.kv_heads = 1;
    p.head_units = rope_dim / 16;
    p.v_units = latent_dim / 16;
    p.pairs = rope_dim / 2;
    p.s_max = s_max;
    p.block_tokens = block_tokens;
    p.max_blocks_per_seq = max_blocks_per_seq;
    p.magnitude = magnitude;
    cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    return type == INSTINFER_F16 ? launch_rope<__half, __half, true>(p, interleaved != 0, stream)
                                 : launch_rope<__nv_bfloat16, __nv_bfloat16, true>(p, interleaved != 0, stream);
}

}  // extern "C"
