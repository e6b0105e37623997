// C ABI, from logits to probabilities: checks and launch.
#include "api_common.cuh"

#include "logits_kernels.cuh"

namespace {

using namespace instinfer;
using namespace instinfer::api;

static_assert(kLogitMaxBias == INSTINFER_MAX_BIAS && kLogitMaxCtas * kLogitThreads * 64 == INSTINFER_MAX_VOCAB, "limits of the header");

// How many clusters of `ctas` blocks the current device holds at once; 0 if it cannot say.  (Asked for once per device,
// kernel, cluster and KiB of the table: the answer takes longer than a small launch.)
int64_t resident_clusters(const void *kernel, unsigned ctas, size_t table)
{
    struct Known {
        const void *kernel;
        unsigned ctas;
        int dev;
        size_t kib;
        int clusters;
    };
    static thread_local Known known[16] = {};
    static thread_local unsigned next = 0;
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess) return 0;
    const size_t kib = (table + 1023) / 1024;
    for (const Known &k : known)
        if (k.kernel == kernel && k.ctas == ctas && k.dev == dev && k.kib == kib) return k.clusters;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(ctas);
    cfg.blockDim = dim3(kLogitThreads);
    cfg.dynamicSmemBytes = kib * 1024;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = ctas;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    int clusters = 0;
    if (cudaOccupancyMaxActiveClusters(&clusters, kernel, &cfg) != cudaSuccess || clusters <= 0) {
        (void)cudaGetLastError();
        return 0;
    }
    known[next++ % 16] = Known{kernel, ctas, dev, kib, clusters};
    return clusters;
}

template <typename E, int kHeld, int kVec>
int launch_logits(const LogitParams &p, int64_t rows, unsigned ctas, size_t table, cudaStream_t stream)
{
    if (table > 40 * 1024) {                   // (beside the kernel's own, more than goes without asking)
        static bool done[kMaxDevices] = {};
        int dev = 0;
        if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= kMaxDevices) return INSTINFER_ERR_CUDA;
        if (!done[dev]) {
            if (cudaFuncSetAttribute(process_logits_kernel<E, kHeld, kVec>, cudaFuncAttributeMaxDynamicSharedMemorySize, kLogitThreads * kHeld * 4) != cudaSuccess) {
                (void)cudaGetLastError();
                return INSTINFER_ERR_CUDA;
            }
            done[dev] = true;
        }
    }
    const int64_t clusters = rows < 2 ? rows : resident_clusters((const void *)process_logits_kernel<E, kHeld, kVec>, ctas, table);
    if (clusters <= 0) return INSTINFER_ERR_CUDA;
    const cudaError_t err = launch_clustered(process_logits_kernel<E, kHeld, kVec>, (unsigned)((rows < clusters ? rows : clusters) * ctas), ctas, kLogitThreads,
                                             table, stream, p);
    return err == cudaSuccess && cudaGetLastError() == cudaSuccess ? INSTINFER_OK : INSTINFER_ERR_CUDA;
}

template <typename E, int kVec>
int launch_logits_held(const LogitParams &p, int64_t rows, unsigned ctas, size_t table, cudaStream_t stream)
{
    const int64_t held = ceil_div(p.slice, kLogitThreads);
    if (held <= 8) return launch_logits<E, 8, kVec>(p, rows, ctas, table, stream);
    if (held <= 16) return launch_logits<E, 16, kVec>(p, rows, ctas, table, stream);
    if (held <= 32) return launch_logits<E, 32, kVec>(p, rows, ctas, table, stream);
    return launch_logits<E, 64, kVec>(p, rows, ctas, table, stream);
}

// Blocks of a row: eight where rows are so few that the GPU has room for them all at once, else as many as leave a
// thread 32 logits at most (64 where eight blocks are not enough for that).
unsigned logit_ctas(int64_t rows, int32_t places)
{
    unsigned ctas = 1;
    const bool few = rows * kLogitMaxCtas <= 2 * (int64_t)sm_count();
    while (ctas < (unsigned)kLogitMaxCtas && places > (int64_t)ctas * kLogitThreads * (few ? 8 : 32)) ctas *= 2;
    return ctas;
}

}  // namespace

extern "C" {

int instinfer_process_logits(void *out, int32_t out_type, int64_t out_stride, const void *logits, int32_t logits_type,
                             int64_t row_stride, const int32_t *tokens, const int32_t *token_lens,
                             const int32_t *prompt_lens, int32_t max_tokens, const float *penalties,
                             const int32_t *draft_tokens, const uint64_t *tree_mask, const int32_t *tree_lens,
                             const int32_t *bias_tokens, const float *bias_values, int32_t max_bias,
                             const uint32_t *allowed, const float *temperatures, int32_t probabilities, int32_t batch,
                             int32_t tree_tokens, int32_t vocab, int32_t *status_flags, void *cuda_stream)
{
    if (batch < 0 || batch > 1 << 24 || tree_tokens <= 0 || vocab <= 0 || max_tokens < 0 || max_bias < 0 || row_stride < vocab || out_stride < vocab)
        return INSTINFER_ERR_INVALID_ARG;
    if (tree_tokens > INSTINFER_MAX_TREE_TOKENS || vocab > INSTINFER_MAX_VOCAB || max_bias > INSTINFER_MAX_BIAS) return INSTINFER_ERR_UNSUPPORTED;
    for (const int32_t type : {out_type, logits_type})
        if (type != INSTINFER_F32 && type != INSTINFER_F16 && type != INSTINFER_BF16) return INSTINFER_ERR_UNSUPPORTED;
    if (batch == 0) return INSTINFER_OK;
    if (!usable(out) || !usable(logits) || !aligned16(tree_mask) || (tokens == nullptr && max_tokens > 0) || (bias_tokens != nullptr && bias_values == nullptr))
        return INSTINFER_ERR_INVALID_ARG;
    const int64_t rows = (int64_t)batch * tree_tokens;
    // Input and output rows that start alike between 4-element boundaries are taken four logits at a time.  A row that
    // starts between them has up to three places more, which have to fit too.
    bool alike = (row_stride - out_stride) % 4 == 0;
    const int32_t late = row_stride % 4 == 0 ? 0 : 3;
    if (vocab + late > INSTINFER_MAX_VOCAB) alike = false;
    const int32_t places = vocab + (alike ? late : 0);
    const unsigned ctas = logit_ctas(rows, places);
    if (rows * ctas >= (int64_t)1 << 31) return INSTINFER_ERR_INVALID_ARG;
    LogitParams p = {};
    p.out = out;
    p.logits = logits;
    p.tokens = max_tokens > 0 ? tokens : nullptr;
    p.token_lens = token_lens;
    p.prompt_lens = prompt_lens;
    p.penalties = penalties;
    p.draft_tokens = draft_tokens;
    p.tree_mask = tree_mask;
    p.tree_lens = tree_lens;
    p.bias_tokens = bias_tokens;
    p.bias_values = bias_values;
    p.allowed = allowed;
    p.temperatures = temperatures;
    p.status = status_flags;
    p.row_stride = row_stride;
    p.out_stride = out_stride;
    p.out_type = out_type;
    p.max_tokens = max_tokens;
    p.max_bias = max_bias;
    p.rows = (int32_t)rows;
    p.tree_tokens = tree_tokens;
    p.vocab = vocab;
    p.slice = (int32_t)(ceil_div(ceil_div(places, ctas), 4) * 4);
    p.probabilities = probabilities;
    const size_t table = penalties != nullptr || bias_tokens != nullptr ? (size_t)p.slice * sizeof(unsigned) : 0;
    cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    switch (logits_type) {
    case INSTINFER_F32:
        return alike ? launch_logits_held<float, 4>(p, rows, ctas, table, stream) : launch_logits_held<float, 1>(p, rows, ctas, table, stream);
    case INSTINFER_F16:
        return alike ? launch_logits_held<__half, 4>(p, rows, ctas, table, stream) : launch_logits_held<__half, 1>(p, rows, ctas, table, stream);
    default:
        return alike ? launch_logits_held<__nv_bfloat16, 4>(p, rows, ctas, table, stream) : launch_logits_held<__nv_bfloat16, 1>(p, rows, ctas, table, stream);
    }
}

}  // extern "C"
