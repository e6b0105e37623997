/*
 * instinfer.h -- C ABI of the decode-attention library (sm_100a).
 *
 * One decode step of one transformer layer, per (sequence, head): the newest token's k,v
 * are appended to that sequence's fp16 KV cache, then its single query row computes
 * q.K^T over every cached key, a softmax scaled by `scale`, and the weighted sum of V.
 * This is the work the paper moves into the storage drive together with the KV cache:
 * the decode-phase "Logit" and "Attend" operators (Sec. III-B) of
 * Attention(Q,K,V) = softmax(Q K^T / sqrt(d_k)) V (Sec. II-A) with a KV cache (Sec. II-B).
 *
 * Conventions common to every entry point
 * ---------------------------------------
 * - Every pointer is a DEVICE pointer unless a comment says "host".  Data pointers must be
 *   16-byte aligned.  The library allocates nothing, never synchronises, and only enqueues
 *   work on `cuda_stream` (a cudaStream_t passed as void*; NULL = the default stream).  The
 *   caller owns every buffer, the workspace included, and must keep it alive until the
 *   enqueued work has run.
 * - fp16 = IEEE binary16.  heads = number of attention heads (query heads == KV heads,
 *   multi-head attention, Sec. II-A).  head_dim must be 128 (the paper's head size,
 *   Sec. IV-C); the two appends and instinfer_decode_attention_grouped also take 64 and 256.
 * - seq_lens[b] (int32, device, [batch]) is the length of sequence b AFTER this step's
 *   append: the append writes logical position seq_lens[b]-1, attention covers positions
 *   [0, seq_lens[b]) -- the new token attends to itself (Sec. II-B).  seq_lens[b] == 0
 *   marks an inactive slot: nothing is appended, its output rows are 0 and its lse -inf.
 * - Contiguous layout: K and V caches are [batch, heads, s_max, head_dim], row-major.
 * - Paged layout (the counterpart of the paper's token-indexed page groups, Sec. IV-C):
 *   K pool and V pool are each [num_phys_blocks, heads, block_tokens, head_dim]; logical
 *   token i of sequence b lives in physical block block_table[b][i / block_tokens] at slot
 *   i % block_tokens; block_table is int32 [batch, max_blocks_per_seq], shared by K and V.
 *   Entries past a sequence's last block are never read.  block_tokens must be a positive
 *   multiple of 8.
 * - Cache slots outside [0, seq_lens[b]) are never read and never influence a result.
 * - Return value: an instinfer_status.  Everything the host can check (null or misaligned
 *   pointers, non-positive sizes, unsupported head_dim or block_tokens, a workspace that is
 *   too small) fails before anything is enqueued.  A failed launch gives INSTINFER_ERR_CUDA.
 * - Data-dependent violations are found on the device and never fault it: a bit is OR-ed
 *   into *status_flags (int32, device, nullable; the caller zeroes it and reads it back
 *   when it wants to know).  A sequence whose length is out of range is treated as
 *   inactive (nothing appended, zero output).  A block-table entry outside
 *   [0, num_phys_blocks) is not dereferenced: the append skips that sequence, attention
 *   reads that block's rows as zeros (the sequence's output is then meaningless but finite).
 *   No kernel traps, asserts or waits on another kernel; the only waits inside a kernel are
 *   for its own asynchronous copies, and those give up after a time limit (see
 *   INSTINFER_FLAG_COPY_TIMEOUT).
 * - Stream order is kept: each kernel sees everything enqueued before it on the stream as
 *   complete.  Internally the launches use programmatic dependent launch, so a kernel's
 *   blocks may already be resident while the previous kernel drains; they touch no memory
 *   before that kernel has completed.
 * - batch == 0 is a valid empty call: INSTINFER_OK, nothing enqueued.
 */
#ifndef INSTINFER_H_
#define INSTINFER_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
    INSTINFER_OK = 0,
    INSTINFER_ERR_INVALID_ARG = 1,   /* null / misaligned pointer, non-positive size, bad bound */
    INSTINFER_ERR_UNSUPPORTED = 2,   /* head_dim or block_tokens outside the supported set     */
    INSTINFER_ERR_WORKSPACE = 3,     /* workspace null or smaller than instinfer_workspace_bytes */
    INSTINFER_ERR_CUDA = 4           /* the CUDA runtime refused a launch                        */
} instinfer_status;

/* Element types, where a call takes more than fp16. */
#define INSTINFER_F32 0
#define INSTINFER_F16 1
#define INSTINFER_BF16 2

/* Bits OR-ed into *status_flags by the kernels. */
#define INSTINFER_FLAG_SEQ_LEN_RANGE 1  /* seq_lens[b] < 0, beyond the cache capacity, or beyond max_seq_len */
#define INSTINFER_FLAG_BLOCK_RANGE   2  /* a block_table entry that had to be read lies outside [0, num_phys_blocks) */
#define INSTINFER_FLAG_TREE_RANGE    16 /* draft trees: a tree length, parent, token or path outside its range, or a
                                           distribution without a positive value */
#define INSTINFER_FLAG_POOL          32 /* block pools: too few free blocks, an impossible fork, or reference counts that
                                           do not fit the tables */
#define INSTINFER_FLAG_TOKEN_RANGE   64 /* logits: a token outside the vocabulary, or a history's lengths out of range */
#define INSTINFER_FLAG_BOUNDS_CHECK  8  /* only in the bounds-checking build of the library (compiled with
                                           -DINSTINFER_BOUNDS_CHECK): a kernel computed a global offset outside the
                                           extent that the call's shapes imply and skipped that access; a defect of
                                           the library, never of the caller's data */
#define INSTINFER_FLAG_COPY_TIMEOUT  4  /* an asynchronous copy inside a kernel did not complete within about two
                                           seconds (a hardware problem, never a data problem); the kernel ended
                                           instead of waiting on and the outputs of that call are undefined */

/*
 * Append (Sec. II-B: the new token's k,v join the cache; Sec. IV-C, batch writing of the
 * decode phase's new vectors).  Copies the bit patterns of k_new[b][h][:] and v_new[b][h][:]
 * (fp16 [batch, heads, head_dim]) into logical position seq_lens[b]-1 of the caches.
 *   block_table == NULL : contiguous caches [batch, heads, s_max, head_dim];
 *                         max_blocks_per_seq, block_tokens, num_phys_blocks are ignored.
 *   block_table != NULL : paged pools; s_max is ignored.
 * k_cache / v_cache are the only buffers this call mutates, and only those rows.
 */
int instinfer_kv_append(void *k_cache, void *v_cache,
                        const void *k_new, const void *v_new,
                        const int32_t *seq_lens,
                        const int32_t *block_table, int32_t max_blocks_per_seq,
                        int32_t block_tokens, int64_t num_phys_blocks,
                        int32_t batch, int32_t heads, int32_t head_dim, int32_t s_max,
                        int32_t *status_flags, void *cuda_stream);

/*
 * Bulk append (the prefill phase hands a layer's K,V of all prompt tokens to the cache at
 * once, Sec. IV-D).  Sequence b receives new_lens[b] tokens (0 <= new_lens[b] <= max_new,
 * new_lens[b] <= seq_lens[b]) from k_new / v_new, fp16 [batch, max_new, heads, head_dim]
 * (token-major, as a projection produces them), at logical positions
 * seq_lens[b]-new_lens[b] .. seq_lens[b]-1; seq_lens are the lengths AFTER the append.
 * Layout selection and the other arguments as in instinfer_kv_append.  A sequence whose
 * lengths are out of range is skipped and flagged.
 */
int instinfer_kv_append_bulk(void *k_cache, void *v_cache,
                             const void *k_new, const void *v_new,
                             const int32_t *seq_lens, const int32_t *new_lens,
                             const int32_t *block_table, int32_t max_blocks_per_seq,
                             int32_t block_tokens, int64_t num_phys_blocks,
                             int32_t batch, int32_t max_new, int32_t heads, int32_t head_dim,
                             int32_t s_max, int32_t *status_flags, void *cuda_stream);

/*
 * Decode attention over a contiguous cache (Sec. II-A definition, Sec. II-B/III-B decode
 * form): out[b][h][:] = softmax_i(scale * q[b][h].K[b][h][i]) . V[b][h][i], i < seq_lens[b].
 *   out          fp16 [batch, heads, head_dim]; fp32 accumulation, rounded once (nearest even)
 *   lse          fp32 [batch, heads], nullable: max_i s_i + ln sum_i exp(s_i - max), s = scale*q.k
 *   q            fp16 [batch, heads, head_dim]
 *   max_seq_len  host upper bound on every seq_lens[b], 1 <= max_seq_len <= s_max; a longer
 *                sequence is treated as inactive and flagged
 *   workspace    at least instinfer_workspace_bytes(batch, heads, head_dim, max_seq_len) bytes;
 *                holds the per-split partial outputs between the two kernels; contents are
 *                scratch before and after the call
 */
int instinfer_decode_attention(void *out, float *lse, const void *q,
                               const void *k_cache, const void *v_cache,
                               const int32_t *seq_lens,
                               int32_t batch, int32_t heads, int32_t head_dim,
                               int32_t s_max, int32_t max_seq_len, float scale,
                               void *workspace, size_t workspace_bytes,
                               int32_t *status_flags, void *cuda_stream);

/*
 * The same over block-paged pools with a block table (Sec. IV-C token-indexed groups).
 * max_seq_len <= max_blocks_per_seq * block_tokens.  The split of a sequence into partial
 * results follows logical token positions only, so the result does not depend on which
 * physical blocks hold the tokens.
 */
int instinfer_decode_attention_paged(void *out, float *lse, const void *q,
                                     const void *k_pool, const void *v_pool,
                                     const int32_t *block_table, const int32_t *seq_lens,
                                     int32_t batch, int32_t heads, int32_t head_dim,
                                     int32_t block_tokens, int32_t max_blocks_per_seq,
                                     int64_t num_phys_blocks, int32_t max_seq_len, float scale,
                                     void *workspace, size_t workspace_bytes,
                                     int32_t *status_flags, void *cuda_stream);

/*
 * Decode attention without a caller-supplied workspace (the paper has no counterpart: its
 * engine has no split partials to park).  For callers that have no device memory of their
 * own to hand over and may not ask the driver for any: a serving engine that gave its whole
 * memory budget to the KV pool at start-up, a plug-in that runs under someone else's
 * allocator, a latency-critical loop in which an allocation's implicit device
 * synchronisation is not acceptable.  The partial results live in a 16 MiB array that is
 * part of the library image, so every GPU context that loads the library carries those
 * 16 MiB until it exits.
 *   block_table == NULL : contiguous caches, arguments as instinfer_decode_attention
 *                         (block_tokens, max_blocks_per_seq, num_phys_blocks ignored);
 *   block_table != NULL : paged pools, arguments as instinfer_decode_attention_paged
 *                         (s_max ignored).
 * Results are those of the two entry points above, bit for bit.
 * Limits and rules:
 * - instinfer_workspace_bytes(batch, heads, head_dim, max_seq_len) must not exceed
 *   INSTINFER_STATIC_WORKSPACE_BYTES; otherwise INSTINFER_ERR_WORKSPACE, nothing enqueued.
 * - The first call on each device looks up the array's device address (the device must be
 *   current); make that first call outside any stream capture.  No call allocates or frees.
 * - All calls on a device share the one array, which keeps whatever the last call left in
 *   it.  Nothing in it needs to start at zero: a call only reads back the slots it has
 *   itself just written.  Two calls that can run at the same time on the GPU (different
 *   streams, no dependency between them) race on it and corrupt each other's results:
 *   order them on one stream or with events.
 */
#define INSTINFER_STATIC_WORKSPACE_BYTES ((size_t)16 << 20)
int instinfer_decode_attention_static(void *out, float *lse, const void *q,
                                      const void *k_cache, const void *v_cache,
                                      const int32_t *block_table, const int32_t *seq_lens,
                                      int32_t batch, int32_t heads, int32_t head_dim,
                                      int32_t s_max, int32_t block_tokens,
                                      int32_t max_blocks_per_seq, int64_t num_phys_blocks,
                                      int32_t max_seq_len, float scale,
                                      int32_t *status_flags, void *cuda_stream);

/*
 * Decode attention on one head shard of a multi-GPU deployment, with the all-gather of the
 * outputs fused into the last kernel (Sec. IV-D, "Scale to CSD array": heads are independent,
 * each device keeps the KV cache of its own heads and computes them locally; only the small
 * output vectors are exchanged).  This GPU holds `heads` consecutive heads, global heads
 * head_offset .. head_offset + heads - 1 of total_heads, in caches shaped as for the two
 * single-GPU entry points with H = heads (block_table == NULL: contiguous, else paged).  The
 * kernel that finishes a (sequence, head) writes its output row into EVERY rank's full
 * output buffer at [b, head_offset + h, :], with plain 16-byte stores:
 *   out_all   HOST array of n_ranks DEVICE pointers; entry r is rank r's fp16
 *             [batch, total_heads, head_dim] buffer as addressable from THIS GPU (its own
 *             allocation, or a peer mapping: CUDA IPC, symmetric memory).  The array is read
 *             during the call only.  1 <= n_ranks <= INSTINFER_MAX_RANKS.
 *   lse       nullable, this shard's own [batch, heads] (not exchanged).
 *   workspace at least instinfer_allgather_workspace_bytes(batch, heads, head_dim, max_seq_len).
 * Every other argument as in instinfer_decode_attention / instinfer_decode_attention_paged.
 * No rank waits for another inside the kernels and nothing here synchronises GPUs: when every
 * rank's call has completed, every buffer holds all heads.  Ordering a reader on rank r after
 * the other ranks' calls is the caller's job (an event exchange, or a barrier collective
 * enqueued after the call on each rank's stream).  Errors as for the single-GPU entry points;
 * head_offset < 0 or head_offset + heads > total_heads: INSTINFER_ERR_INVALID_ARG.
 */
#define INSTINFER_MAX_RANKS 16
int instinfer_decode_attention_allgather(void *const *out_all, int32_t n_ranks, float *lse,
                                         const void *q, const void *k_cache, const void *v_cache,
                                         const int32_t *block_table, const int32_t *seq_lens,
                                         int32_t batch, int32_t heads, int32_t head_offset,
                                         int32_t total_heads, int32_t head_dim, int32_t s_max,
                                         int32_t block_tokens, int32_t max_blocks_per_seq,
                                         int64_t num_phys_blocks, int32_t max_seq_len, float scale,
                                         void *workspace, size_t workspace_bytes,
                                         int32_t *status_flags, void *cuda_stream);

size_t instinfer_allgather_workspace_bytes(int32_t batch, int32_t heads, int32_t head_dim,
                                           int32_t max_seq_len);

/*
 * Decode attention for configurations other than the paper's one query head per KV head and
 * one new token per step (Sec. II-A, II-B; Sec. IV-C only notes that other configurations
 * exist): grouped heads, several new tokens per step, head sizes 64 / 128 / 256.
 *   q, out   fp16 [batch, q_tokens, q_heads, head_dim]
 *   lse      nullable fp32 [batch, q_tokens, q_heads]
 *   caches   as for the entry points above with `kv_heads` heads (block_table == NULL:
 *            contiguous [batch, kv_heads, s_max, head_dim], else paged pools
 *            [num_phys_blocks, kv_heads, block_tokens, head_dim])
 * Query head hq reads KV head hq / (q_heads / kv_heads); q_heads must be a multiple of
 * kv_heads.  The caches already hold all q_tokens new tokens (append them with
 * instinfer_kv_append, or instinfer_kv_append_bulk for q_tokens > 1) and seq_lens[b] counts
 * them; new token t (0 = oldest) attends causally to positions
 * [0, seq_lens[b] - (q_tokens - 1 - t)).  A token whose range is empty gives a zero row and
 * lse = -inf.  With q_tokens = 1 and q_heads = kv_heads the result is that of the entry points
 * above within the same tolerance (not bit for bit: the contractions run on the tensor cores).
 * Limits (INSTINFER_ERR_UNSUPPORTED otherwise): (q_heads / kv_heads) * q_tokens <= 16;
 * head_dim in {64, 128, 256}; paged block_tokens a multiple of 16.  Scaled logits from some 9e7 on (2^27 to
 * the base 2) may overflow the weights, to NaN; instinfer_decode_attention_tree has no such limit.
 *   workspace at least instinfer_grouped_workspace_bytes(...) bytes.
 */
int instinfer_decode_attention_grouped(void *out, float *lse, const void *q, const void *k_cache,
                                       const void *v_cache, const int32_t *block_table,
                                       const int32_t *seq_lens, int32_t batch, int32_t q_tokens,
                                       int32_t q_heads, int32_t kv_heads, int32_t head_dim,
                                       int32_t s_max, int32_t block_tokens,
                                       int32_t max_blocks_per_seq, int64_t num_phys_blocks,
                                       int32_t max_seq_len, float scale, void *workspace,
                                       size_t workspace_bytes, int32_t *status_flags,
                                       void *cuda_stream);

size_t instinfer_grouped_workspace_bytes(int32_t batch, int32_t q_tokens, int32_t q_heads,
                                         int32_t kv_heads, int32_t head_dim, int32_t max_seq_len);

/*
 * ---- Rotary positions on the way into the cache ----
 * (No counterpart in the paper, whose models have learned positions.)  Queries and keys of models with rotary
 * positions are turned by their position before they are used: with pairs (a_i, b_i) of a head's first rope_dim dims,
 *     (a_i, b_i) -> magnitude * (a_i cos t - b_i sin t, a_i sin t + b_i cos t),  t = position * frequencies[i],
 * i < rope_dim / 2; pair i is dims (i, rope_dim / 2 + i) (halves), or (2 i, 2 i + 1) (interleaved != 0).  The other dims stay.
 * The angle is computed in 64 bits (so that far positions keep their fast pairs), the turn in 32, rounded once.
 *
 * instinfer_rope_frequencies: the pairs' frequencies and the magnitude, HOST memory, host computation only.
 *   plain     f_i = base^(-2 i / rope_dim), magnitude 1
 *   linear    f_i / factor, magnitude 1 (positions squeezed into the trained range)
 *   by parts  for a context stretched `factor` times beyond trained_len: pairs that turn at least fast_turns times over
 *             trained_len tokens keep f_i, those that turn at most slow_turns times get f_i / factor, between them linearly
 *             (in the number of turns); magnitude 0.1 ln(factor) + 1
 * factor >= 1; trained_len > 0 and 0 <= slow_turns < fast_turns are looked at for "by parts" only.
 * rope_dim is positive and even.  An unknown scaling: INSTINFER_ERR_UNSUPPORTED.
 */
#define INSTINFER_ROPE_PLAIN 0
#define INSTINFER_ROPE_LINEAR 1
#define INSTINFER_ROPE_BY_PARTS 2
int instinfer_rope_frequencies(double *frequencies, float *magnitude, int32_t rope_dim, double base,
                               int32_t scaling, double factor, int32_t trained_len, double slow_turns,
                               double fast_turns);

/*
 * What instinfer_kv_append_bulk does, with the keys turned on the way, and the queries turned in the same pass.
 * Sequence b receives new_lens[b] tokens (new_lens == NULL: max_new tokens each, none for a sequence of length 0) at
 * logical positions seq_lens[b] - new_lens[b] .. seq_lens[b] - 1 of the cache.
 *   q_out      fp16 [batch, max_new, q_heads, head_dim], turned (what the attention calls take); rows of tokens that there
 *              are not stay as they were.  May be q itself where type is fp16 and q_stride = q_heads * head_dim.
 *   q, k_new, v_new  `type` (INSTINFER_F32, _F16 or _BF16), token (b, t) at (b * max_new + t) * stride elements, its heads
 *              one after the other (so all three may be slices of one projection's output).  Strides are multiples of
 *              16 bytes.  q_heads == 0: q and q_out are not looked at.
 *   frequencies  fp64 [rope_dim / 2], DEVICE, radians per position; 8-byte aligned
 *   positions  nullable int32 [batch, max_new]: the positions to turn by (any value; a draft tree's nodes, say, whose
 *              depth is not their place in the cache).  NULL: the logical positions in the cache.
 * fp32 and bf16 values are rounded to fp16 once (values beyond its range become infinities); fp16 values and keys' other dims are
 * bit copies.  Layout selection and the other arguments as in instinfer_kv_append_bulk.  A sequence whose lengths are out of
 * range is skipped and flagged; a token whose block is out of range is flagged, its K and V rows are not written.
 * Limits (INSTINFER_ERR_UNSUPPORTED otherwise): head_dim in {64, 128, 256}, rope_dim a multiple of 16.
 */
int instinfer_rope_append(void *q_out, void *k_cache, void *v_cache, const void *q, const void *k_new,
                          const void *v_new, int32_t type, int64_t q_stride, int64_t k_stride,
                          int64_t v_stride, const double *frequencies, int32_t rope_dim,
                          int32_t interleaved, float magnitude, const int32_t *positions,
                          const int32_t *seq_lens, const int32_t *new_lens, const int32_t *block_table,
                          int32_t max_blocks_per_seq, int32_t block_tokens, int64_t num_phys_blocks,
                          int32_t batch, int32_t max_new, int32_t q_heads, int32_t kv_heads,
                          int32_t head_dim, int32_t s_max, int32_t *status_flags, void *cuda_stream);

/*
 * ---- A cache of one latent vector a token ----
 * (No counterpart in the paper, whose models have keys and values for every head.)  Models with latent attention cache one
 * vector of latent_dim values a token, from which the keys and values of all heads are made, and a key part of rope_dim
 * dims with rotary position that all heads share.  In decoding the matrices that make them are absorbed by the queries
 * and the outputs, so that a head's query is a vector of latent_dim + rope_dim values, the cache row is every head's key,
 * and its first latent_dim values are every head's value:
 *     out[r] = softmax_i(scale * q[r] . row_i) . row_i[0 .. latent_dim)
 * Layouts: contiguous [batch, s_max, latent_dim + rope_dim], or a pool [num_phys_blocks, block_tokens, latent_dim + rope_dim]
 * with a block table; fp16 or bf16 (`type`, the same for every tensor of a call but lse).
 * The calls that move rows and blocks (instinfer_kv_keep_path, instinfer_kv_fork, instinfer_kv_resize, instinfer_kv_defragment) take
 * such caches as caches of one head of latent_dim + rope_dim, half of the layers as K and half as V caches; with an odd number
 * of layers one of them stands in both lists, at the same place (instinfer_kv_keep_path refuses one that stands at two places).
 * Limits (INSTINFER_ERR_UNSUPPORTED otherwise): latent_dim 512, rope_dim 64; paged block_tokens a multiple of 8.
 *
 * instinfer_latent_append: the new tokens' rows, with the key part turned, and the queries' turned parts.
 *   q_out      [batch, max_new, q_heads, latent_dim + rope_dim], the absorbed queries: the last rope_dim values of the rows of
 *              tokens that there are get written, nothing else
 *   q_rope     the queries' parts to turn, token (b, t) and head h at (b * max_new + t) * q_stride + h * q_head_stride elements
 *              (token after token or head after head; they must not overlap)
 *   latent_new, rope_new  token (b, t) at (b * max_new + t) * stride elements; strides are multiples of 16 bytes
 * frequencies [rope_dim / 2] and all else as in instinfer_rope_append.
 */
int instinfer_latent_append(void *q_out, void *cache, const void *q_rope, const void *latent_new,
                            const void *rope_new, int32_t type, int64_t q_stride, int64_t q_head_stride,
                            int64_t latent_stride, int64_t rope_stride, const double *frequencies,
                            int32_t interleaved, float magnitude, const int32_t *positions,
                            const int32_t *seq_lens, const int32_t *new_lens, const int32_t *block_table,
                            int32_t max_blocks_per_seq, int32_t block_tokens, int64_t num_phys_blocks,
                            int32_t batch, int32_t max_new, int32_t q_heads, int32_t latent_dim,
                            int32_t rope_dim, int32_t s_max, int32_t *status_flags, void *cuda_stream);

/*
 * Decode attention over a latent cache, for one new token, several, or a draft tree (see below).
 *   q          [batch, q_tokens, q_heads, latent_dim + rope_dim], absorbed queries with their parts turned
 *   out        [batch, q_tokens, q_heads, latent_dim]; fp32 accumulation, rounded once
 *   lse        nullable fp32 [batch, q_tokens, q_heads]
 *   tree_lens  nullable int32 [batch]: how many of the q_tokens new tokens there are (NULL: all); they are the last
 *              tree_lens[b] positions of the sequence, and the caches hold them
 *   tree_mask  NULL: new token t attends to the positions up to its own.  Else as instinfer_tree_mask writes it, 16-byte
 *              aligned: to every position before the new ones and to the new ones whose bits its row has.
 *   workspace  at least instinfer_latent_workspace_bytes(...) bytes
 * Rows of new tokens that there are not, rows that see nothing, and all rows of a sequence with seq_lens[b] == 0 are zero
 * with lse = -inf.  A tree_lens[b] out of range or above seq_lens[b] is flagged (INSTINFER_FLAG_TREE_RANGE) and makes the
 * sequence inactive.  What a row does not see never influences it, infinities and NaN in hidden new tokens' rows
 * included.  A row that sees a token whose values make its logit NaN or +infinity becomes NaN.  A token whose logit is
 * -infinity counts nothing; the dims in which its vector is infinite may become NaN if it is not one of the new
 * tokens.  Block-table entries out of range count as rows of zeros (flagged).
 * Limits (INSTINFER_ERR_UNSUPPORTED otherwise): q_tokens <= INSTINFER_MAX_TREE_TOKENS, q_tokens * q_heads <=
 * INSTINFER_MAX_LATENT_ROWS, caches of fewer than 2^31 rows.
 */
#define INSTINFER_MAX_LATENT_ROWS 16384
int instinfer_decode_attention_latent(void *out, float *lse, const void *q, const void *cache,
                                      const int32_t *block_table, const int32_t *seq_lens,
                                      const int32_t *tree_lens, const uint64_t *tree_mask, int32_t type,
                                      int32_t batch, int32_t q_tokens, int32_t q_heads,
                                      int32_t latent_dim, int32_t rope_dim, int32_t s_max,
                                      int32_t block_tokens, int32_t max_blocks_per_seq,
                                      int64_t num_phys_blocks, int32_t max_seq_len, float scale,
                                      void *workspace, size_t workspace_bytes, int32_t *status_flags,
                                      void *cuda_stream);

size_t instinfer_latent_workspace_bytes(int32_t batch, int32_t q_tokens, int32_t q_heads,
                                        int32_t latent_dim, int32_t rope_dim, int32_t max_seq_len);

/*
 * ---- Speculative decoding: several drafted tokens per sequence and step ----
 * (No counterpart in the paper, whose decode phase adds one token per step, Sec. II-B; the work
 * stays its Logit / Attend operators, Sec. III-B, over the same cache.)
 *
 * A draft tree has tree_lens[b] nodes (0 <= tree_lens[b] <= tree_tokens; tree_lens == NULL:
 * tree_tokens each).  Node 0 is its root, the newest token that is certain; a node comes after
 * its parent.  The caches hold all nodes behind the sequence's other tokens, node j at position
 * seq_lens[b] - tree_lens[b] + j (append them with instinfer_kv_append_bulk); seq_lens[b] counts
 * them.  One step is: make room (instinfer_kv_resize), append, instinfer_tree_mask once, in every
 * layer instinfer_decode_attention_tree, then instinfer_verify_tree, instinfer_kv_keep_path, and
 * instinfer_kv_resize to the kept length.  On a paged cache the step needs blocks of a multiple of 16
 * tokens, which the attention asks for (the other calls take multiples of 8).
 * Limit (INSTINFER_ERR_UNSUPPORTED otherwise): tree_tokens <= INSTINFER_MAX_TREE_TOKENS.
 */
#define INSTINFER_MAX_TREE_TOKENS 128

/*
 * Which nodes a node sees: itself and its ancestors.
 *   tree_mask  uint64 [batch, tree_tokens, W], W = (tree_tokens + 63) / 64: bit j % 64 of word
 *              j / 64 of row t is set if node t sees node j; rows from tree_lens[b] on are 0
 *   parents    int32 [batch, tree_tokens]: parents[b][t] < t, -1 for a root.  Any other value is
 *              flagged (INSTINFER_FLAG_TREE_RANGE) and taken for -1; a tree_lens[b] out of range
 *              is flagged and taken for 0.
 */
int instinfer_tree_mask(uint64_t *tree_mask, const int32_t *parents, const int32_t *tree_lens,
                        int32_t batch, int32_t tree_tokens, int32_t *status_flags, void *cuda_stream);

/*
 * Attention of a tree of drafted tokens over the cache: node t of sequence b attends to every
 * position before the tree and to the nodes whose bits its row of tree_mask has (any mask will do;
 * bits of nodes from tree_lens[b] on are ignored).
 *   q, out     fp16 [batch, tree_tokens, q_heads, head_dim]; grouped heads as in
 *              instinfer_decode_attention_grouped
 *   lse        nullable fp32 [batch, tree_tokens, q_heads]
 *   caches     as for instinfer_decode_attention_grouped (block_table == NULL: contiguous)
 *   tree_mask  as instinfer_tree_mask writes it, 16-byte aligned
 *   workspace  at least instinfer_tree_workspace_bytes(...) bytes
 * Rows of nodes from tree_lens[b] on, rows that see nothing, and all rows of a sequence with
 * seq_lens[b] == 0 are zero with lse = -inf.  A tree_lens[b] out of range or above seq_lens[b] is
 * flagged (INSTINFER_FLAG_TREE_RANGE) and makes the sequence inactive.  What a row does not see
 * never influences it, infinities and NaN in hidden nodes' keys and values included; a NaN that
 * it sees makes the row NaN, an infinity in the rows before the tree makes it infinite or NaN.
 * Limits (INSTINFER_ERR_UNSUPPORTED otherwise): head_dim in {64, 128, 256}; paged block_tokens a
 * multiple of 16; (q_heads / kv_heads) * tree_tokens <= INSTINFER_MAX_TREE_ROWS.
 */
#define INSTINFER_MAX_TREE_ROWS 4096
int instinfer_decode_attention_tree(void *out, float *lse, const void *q, const void *k_cache,
                                    const void *v_cache, const int32_t *block_table,
                                    const int32_t *seq_lens, const int32_t *tree_lens,
                                    const uint64_t *tree_mask, int32_t batch, int32_t tree_tokens,
                                    int32_t q_heads, int32_t kv_heads, int32_t head_dim,
                                    int32_t s_max, int32_t block_tokens,
                                    int32_t max_blocks_per_seq, int64_t num_phys_blocks,
                                    int32_t max_seq_len, float scale, void *workspace,
                                    size_t workspace_bytes, int32_t *status_flags,
                                    void *cuda_stream);

size_t instinfer_tree_workspace_bytes(int32_t batch, int32_t tree_tokens, int32_t q_heads,
                                      int32_t kv_heads, int32_t head_dim, int32_t max_seq_len);

/*
 * Verification of a draft tree against the target's probabilities from given random numbers
 * (recursive rejection sampling).  With p_v and q_v the target's and the draft's distribution after
 * node v, the walk starts at the root; at a node v, w = p_v and Z = 1, and v's children c are tried
 * in index order: c is taken if
 *     uniforms[b][c] * q_v(token_c) * Z < w(token_c),
 * and the walk goes on at c; otherwise w <- max(w - Z q_v, 0) and Z <- sum w (if that sum is 0, w
 * and Z stay as they were).  When no child is taken the next token is the lowest i with
 * w_0 + ... + w_i > uniforms[b][0] * sum w.  Computed in 64 bits.  If v's children were drawn
 * independently from q_v and the rows of p and q sum to 1, the emitted tokens have the target's
 * distribution; as nothing is normalised here, it holds up to what the rows' sums are off by (bf16 and
 * fp16 rows: their rounding).
 *   path        int32 [batch, tree_tokens]: the nodes taken, ascending, the root first; -1 behind
 *   path_lens   int32 [batch]: how many, 0 for a sequence without a tree
 *   out_tokens  int32 [batch, tree_tokens]: the tokens of path[1 ..], then the next token; -1 behind
 *   target_probs, draft_probs  probs_type [batch, tree_tokens, vocab], row t the distributions
 *               after node t, rows row_stride >= vocab elements apart, 16-byte aligned (rows need not
 *               be).  Not normalised here; a value that is not positive and finite counts as 0.
 *               draft_probs == NULL: drafts that were not sampled (q_v is one-hot at token_c).
 *   tokens, parents  int32 [batch, tree_tokens]; a node (other than the root) whose parent is not
 *               an earlier node or whose token is outside [0, vocab) is flagged
 *               (INSTINFER_FLAG_TREE_RANGE) and never taken
 *   uniforms    fp32 [batch, tree_tokens] in [0, 1)
 * If w has no positive value the next token is -1, flagged.
 */
int instinfer_verify_tree(int32_t *path, int32_t *path_lens, int32_t *out_tokens,
                          const void *target_probs, const void *draft_probs, int32_t probs_type,
                          int64_t row_stride, const int32_t *tokens, const int32_t *parents,
                          const int32_t *tree_lens, const float *uniforms, int32_t batch,
                          int32_t tree_tokens, int32_t vocab, int32_t *status_flags,
                          void *cuda_stream);

/*
 * From the logits of a step to the probabilities that instinfer_verify_tree (or any sampling) takes: penalties for repeated
 * tokens, biases, a grammar's mask, the temperature.  For row t of sequence b and token i, in 32 bits, in this order:
 *     token in the sequence's prompt or output:  z = z > 0 ? z / repetition : z * repetition
 *     z -= frequency * n + (n > 0 ? presence : 0),  n = how often the token is in the output
 *     z += the sum of the sequence's biases of the token, in the list's order
 *     token not allowed:  z = -infinity
 *     probability = exp((z - max z) / T) / sum exp((z - max z) / T);  T = 0 (or less): 1 at the largest z, at the lowest
 *     token of equal ones, 0 elsewhere
 * What is not allowed never counts, whatever its logit.  A row in which nothing is left is all zeros (instinfer_verify_tree then
 * flags it and gives -1); an allowed NaN or +infinity makes a row of T > 0 NaN; a NaN is never the largest.
 *   out          out_type [batch, tree_tokens, vocab], rows out_stride >= vocab elements apart; may be logits itself where types and
 *                strides are alike.  Rows of nodes from tree_lens[b] on stay as they were.
 *   logits       logits_type [batch, tree_tokens, vocab], rows row_stride apart.  Either type INSTINFER_F32, _F16 or _BF16.
 *   tokens       nullable int32 [batch, max_tokens]: the sequence's history, the first token_lens[b] (NULL: max_tokens) of them,
 *                of which the first prompt_lens[b] (NULL: 0) are its prompt and the others its output
 *   penalties    nullable fp32 [batch, 3]: repetition (1: none, positive), frequency (0: none), presence (0: none).  NULL: none, and
 *                tokens and draft_tokens are not looked at.
 *   draft_tokens nullable int32 [batch, tree_tokens]: a draft tree's tokens, which are not in `tokens`; those of the nodes that
 *                tree_mask (as instinfer_tree_mask writes it; NULL: a chain) shows to node t are output too for row t
 *   tree_lens    nullable int32 [batch]: rows that there are (NULL: tree_tokens)
 *   bias_tokens, bias_values  nullable int32, fp32 [batch, max_bias]; a negative token is an unused entry
 *   allowed      nullable uint32 [batch, tree_tokens, (vocab + 31) / 32]: bit i % 32 of word i / 32 allows token i
 *   temperatures nullable fp32 [batch], finite (NULL: 1)
 *   probabilities  0: out gets z / T instead (z where T is 0 or less), -infinity where not allowed
 * Tokens >= vocab, tokens of the history or a draft < 0, and lengths out of range are flagged (INSTINFER_FLAG_TOKEN_RANGE;
 * INSTINFER_FLAG_TREE_RANGE for tree_lens, whose rows are then left) and count nothing.
 * Limits (INSTINFER_ERR_UNSUPPORTED otherwise): vocab <= INSTINFER_MAX_VOCAB, max_bias <= INSTINFER_MAX_BIAS, tree_tokens <=
 * INSTINFER_MAX_TREE_TOKENS.
 */
#define INSTINFER_MAX_VOCAB 262144
#define INSTINFER_MAX_BIAS 256
int instinfer_process_logits(void *out, int32_t out_type, int64_t out_stride, const void *logits,
                             int32_t logits_type, int64_t row_stride, const int32_t *tokens,
                             const int32_t *token_lens, const int32_t *prompt_lens, int32_t max_tokens,
                             const float *penalties, const int32_t *draft_tokens,
                             const uint64_t *tree_mask, const int32_t *tree_lens,
                             const int32_t *bias_tokens, const float *bias_values, int32_t max_bias,
                             const uint32_t *allowed, const float *temperatures, int32_t probabilities,
                             int32_t batch, int32_t tree_tokens, int32_t vocab, int32_t *status_flags,
                             void *cuda_stream);

/*
 * Keeps the accepted path of a draft tree in the caches of all layers: the K and V rows of node
 * path[b][i] move from position P + path[b][i] to P + i, P = seq_lens[b] - tree_lens[b], for
 * i < path_lens[b], and new_lens[b] = P + path_lens[b].  Bit copies; only those rows change.
 *   k_caches, v_caches  HOST arrays of n_layers DEVICE pointers, read during the call only; all
 *              layers have the same shape and share seq_lens and block_table
 *   path       ascending node numbers (as instinfer_verify_tree writes them)
 *   new_lens   int32 [batch], a buffer of its own (not seq_lens)
 * Layout selection and the other arguments as in instinfer_kv_append.  A path or tree out of range
 * is flagged (INSTINFER_FLAG_TREE_RANGE, or INSTINFER_FLAG_SEQ_LEN_RANGE for the length), the
 * sequence is left alone and new_lens[b] = seq_lens[b].
 * Limits (INSTINFER_ERR_UNSUPPORTED otherwise): n_layers <= INSTINFER_MAX_LAYERS, head_dim in {64, 128, 256}, or a latent
 * cache's row as one head.
 */
#define INSTINFER_MAX_LAYERS 128
int instinfer_kv_keep_path(void *const *k_caches, void *const *v_caches, int32_t n_layers,
                           const int32_t *path, const int32_t *path_lens, const int32_t *tree_lens,
                           const int32_t *seq_lens, int32_t *new_lens, const int32_t *block_table,
                           int32_t max_blocks_per_seq, int32_t block_tokens, int64_t num_phys_blocks,
                           int32_t batch, int32_t tree_tokens, int32_t heads, int32_t head_dim,
                           int32_t s_max, int32_t *status_flags, void *cuda_stream);

/*
 * ---- Blocks of a paged pool that sequences share ----
 * The state of a pool is block_refs, int32 [num_phys_blocks]: how many sequences' tables list a
 * block, 0 for a free one.  Sequence b lists the blocks of its seq_lens[b] tokens, the first
 * (seq_lens[b] + block_tokens - 1) / block_tokens entries of its row of block_table.  The three
 * calls below keep both in step; all are deterministic (an allocation takes the lowest free ids).
 * They must not run at the same time on one pool.  Arguments as in instinfer_kv_append, layers'
 * pools as in instinfer_kv_keep_path.
 * Limits (INSTINFER_ERR_UNSUPPORTED otherwise): batch <= 8192, batch * max_blocks_per_seq <= 2^28,
 * n_layers <= INSTINFER_MAX_LAYERS, head_dim in {64, 128, 256} or a latent cache's row as one head.
 *
 * instinfer_kv_fork: sequence dst[i] (empty: length 0) becomes a copy of src[i] that shares all of
 * its blocks, the partly filled last one included; nothing is copied but table entries.
 *   src, dst   int32 [n_forks], device; n_forks <= batch.  One source may be forked many times; a
 *              destination may be listed once (later ones are flagged and skipped) and may not be
 *              a source (flagged and skipped).  INSTINFER_FLAG_POOL; a destination that is not empty:
 *              INSTINFER_FLAG_SEQ_LEN_RANGE, skipped.
 */
int instinfer_kv_fork(int32_t *block_table, int32_t *block_refs, int32_t *seq_lens,
                      const int32_t *src, const int32_t *dst, int32_t n_forks,
                      int32_t max_blocks_per_seq, int32_t block_tokens, int64_t num_phys_blocks,
                      int32_t batch, int32_t *status_flags, void *cuda_stream);

/*
 * instinfer_kv_resize: sequence b goes from seq_lens[b] to want_lens[b] tokens (0 frees it).  First
 * shorter sequences give blocks back, then growing ones get blocks, in the order of b.  A growing
 * sequence whose last block is partly filled and also listed by others gets a copy of that block in
 * all layers (copy on write: it is going to write there); if all that list it grow in this call, the
 * last of them keeps the original.  So after the call positions seq_lens[b] .. want_lens[b] - 1 can
 * be appended to without touching another sequence.
 *   new_lens   int32 [batch]: want_lens[b], or seq_lens[b] where the sequence was left as it is; may
 *              be seq_lens or want_lens itself
 * When the free blocks do not suffice for a sequence, it and every later one that needs blocks (or
 * that would keep a shared block) is left as it is, flagged INSTINFER_FLAG_POOL.  Lengths outside
 * [0, max_blocks_per_seq * block_tokens] are flagged and left.
 *   workspace  at least instinfer_kv_resize_workspace_bytes(batch, num_phys_blocks) bytes
 */
int instinfer_kv_resize(void *const *k_pools, void *const *v_pools, int32_t n_layers,
                        int32_t *block_table, int32_t *block_refs, const int32_t *seq_lens,
                        const int32_t *want_lens, int32_t *new_lens, int32_t max_blocks_per_seq,
                        int32_t block_tokens, int64_t num_phys_blocks, int32_t batch, int32_t heads,
                        int32_t head_dim, void *workspace, size_t workspace_bytes,
                        int32_t *status_flags, void *cuda_stream);

size_t instinfer_kv_resize_workspace_bytes(int32_t batch, int64_t num_phys_blocks);

/*
 * instinfer_kv_defragment: the U blocks in use get the ids 0 .. U-1: those with an id of U or more, in
 * ascending order, are copied (in all layers) to the free ids below U, in ascending order; the others
 * stay.  Tables and counts are written to new_block_table [batch, max_blocks_per_seq] and
 * new_block_refs [num_phys_blocks] (which may be block_table and block_refs themselves; entries
 * behind a sequence's last block are copied as they are), *blocks_used = U (device).  Blocks from U
 * on are free afterwards.  A listed block that counts as free is nobody's, and another one may be moved
 * over it: its entries are copied as they are and flagged INSTINFER_FLAG_POOL.  With batch == 0 nothing
 * is enqueued, as everywhere, and nothing is written.
 *   workspace  at least instinfer_kv_defragment_workspace_bytes(num_phys_blocks) bytes
 */
int instinfer_kv_defragment(void *const *k_pools, void *const *v_pools, int32_t n_layers,
                            const int32_t *block_table, int32_t *new_block_table,
                            const int32_t *block_refs, int32_t *new_block_refs,
                            const int32_t *seq_lens, int32_t *blocks_used,
                            int32_t max_blocks_per_seq, int32_t block_tokens,
                            int64_t num_phys_blocks, int32_t batch, int32_t heads, int32_t head_dim,
                            void *workspace, size_t workspace_bytes, int32_t *status_flags,
                            void *cuda_stream);

size_t instinfer_kv_defragment_workspace_bytes(int64_t num_phys_blocks);

/*
 * One whole decode step for a caller whose new vectors live in host memory (the paper's
 * decode flow, Sec. IV-D: only q, k, v travel to the device that owns the KV cache and only
 * the attention output travels back; the cache never moves).
 *   qkv_host  HOST (pinned for an asynchronous copy) fp16 [3, batch, heads, head_dim]:
 *             q, k_new, v_new packed in this order
 *   out_host  HOST fp16 [batch, heads, head_dim]
 *   qkv_dev, out_dev  DEVICE staging buffers of the same shapes, owned by the caller
 *   lse       DEVICE fp32 [batch, heads], nullable
 * Enqueued on the stream, in order: copy qkv_host -> qkv_dev, instinfer_kv_append,
 * instinfer_decode_attention (block_table == NULL) or instinfer_decode_attention_paged,
 * copy out_dev -> out_host.  out_host holds the result once the stream has reached that
 * point; the call itself does not synchronise.  Other arguments and errors as in the calls
 * it is made of.
 */
int instinfer_decode_step_host(void *out_host, const void *qkv_host, void *qkv_dev, void *out_dev,
                               float *lse, void *k_cache, void *v_cache, const int32_t *seq_lens,
                               const int32_t *block_table, int32_t max_blocks_per_seq,
                               int32_t block_tokens, int64_t num_phys_blocks,
                               int32_t batch, int32_t heads, int32_t head_dim, int32_t s_max,
                               int32_t max_seq_len, float scale,
                               void *workspace, size_t workspace_bytes,
                               int32_t *status_flags, void *cuda_stream);

/*
 * The same step with the two copies taken off the compute stream, so that a caller with
 * several independent steps in flight (the paper's mini-batches, Sec. IV-D: one mini-batch's
 * vectors travel while another's attention runs) overlaps the next step's upload and the
 * previous step's download with this step's kernels.  Streams and events are the caller's (cudaStream_t / cudaEvent_t as void*):
 *   upload_stream:    copy qkv_host -> qkv_dev, then record uploaded_event
 *   compute_stream:   wait for uploaded_event, instinfer_kv_append, attention, record attended_event
 *   download_stream:  wait for attended_event, copy out_dev -> out_host
 * A copy stream may be the compute stream itself (then its event is not used and may be
 * NULL); otherwise its event must not be NULL.  Nothing else orders the three streams: the
 * caller keeps qkv_dev, out_dev, the workspace and the events of a call untouched until that
 * call's part of each stream has run (one set per call in flight), and if the streams are
 * being captured into a graph it forks the copy streams from the capturing stream before the
 * first call and joins them after the last.  out_host holds the result once download_stream
 * has reached that point.  Arguments and errors otherwise as instinfer_decode_step_host.
 */
int instinfer_decode_step_host_overlapped(void *out_host, const void *qkv_host, void *qkv_dev, void *out_dev,
                                          float *lse, void *k_cache, void *v_cache, const int32_t *seq_lens,
                                          const int32_t *block_table, int32_t max_blocks_per_seq,
                                          int32_t block_tokens, int64_t num_phys_blocks,
                                          int32_t batch, int32_t heads, int32_t head_dim, int32_t s_max,
                                          int32_t max_seq_len, float scale,
                                          void *workspace, size_t workspace_bytes, int32_t *status_flags,
                                          void *compute_stream, void *upload_stream, void *download_stream,
                                          void *uploaded_event, void *attended_event);

/*
 * ---- Sparse decode attention (the paper's Algorithm 1, SparF; SparQ's arithmetic) ----
 * Paged layout only.  Besides the K and V pools the cache keeps
 *   kt_pool  fp16 [num_kt_blocks, heads, head_dim, kt_block_tokens]: K a second time,
 *            embedding-major inside each block (Sec. IV-C, hidden-embedding-indexed copy).
 *            It has its own block size and its own table kt_block_table
 *            [batch, kt_max_blocks_per_seq]: token i of sequence b is column
 *            i % kt_block_tokens of block kt_block_table[b][i / kt_block_tokens].  As in the
 *            paper, where this mapping uses far larger token groups than the 16-token pages
 *            of K and V, a larger kt_block_tokens (a positive multiple of 8; 128-512 is a good
 *            choice) makes the r selected rows of a block long contiguous runs.  Slots past a
 *            sequence's end inside its last block may be read (in groups of 8 tokens) but
 *            never influence a result;
 *   v_sum    fp32 [batch, heads, head_dim]: the sum of all cached V rows of each sequence;
 *            Algorithm 1's mean value vector is v_sum / seq_lens[b].
 *
 * instinfer_sparf_append does what instinfer_kv_append does on the paged pools and also
 * writes k_new into kt_pool and adds v_new to v_sum (one fp32 rounding per element).
 * seq_lens[b] must fit both tables (max_blocks_per_seq * block_tokens and
 * kt_max_blocks_per_seq * kt_block_tokens); a longer one is flagged and that sequence is left
 * untouched, as is one whose block id in either table is out of range.
 * Unlike the plain append this call is not idempotent: v_sum grows by v_new every time, so
 * replaying a step (a retried request, a benchmark loop) adds the token's value again.
 */
int instinfer_sparf_append(void *k_pool, void *v_pool, void *kt_pool, float *v_sum,
                           const void *k_new, const void *v_new, const int32_t *seq_lens,
                           const int32_t *block_table, int32_t max_blocks_per_seq,
                           int32_t block_tokens, int64_t num_phys_blocks,
                           const int32_t *kt_block_table, int32_t kt_max_blocks_per_seq,
                           int32_t kt_block_tokens, int64_t num_kt_blocks,
                           int32_t batch, int32_t heads, int32_t head_dim,
                           int32_t *status_flags, void *cuda_stream);

/*
 * Bulk form of instinfer_sparf_append for the prefill phase (Sec. IV-D): new_lens[b] tokens
 * per sequence from token-major k_new / v_new [batch, max_new, heads, head_dim], as in
 * instinfer_kv_append_bulk; v_sum receives the tokens in order, one fp32 rounding each, so
 * the result equals that of appending them one by one.  A sequence with a block id out of
 * range among the blocks its new tokens need keeps its transposed copy and its v_sum, but its
 * K and V rows in valid blocks may already have been written: after a flagged call the cache
 * state of the flagged sequence is undefined and the caller should rebuild or drop it.
 */
int instinfer_sparf_append_bulk(void *k_pool, void *v_pool, void *kt_pool, float *v_sum,
                                const void *k_new, const void *v_new, const int32_t *seq_lens,
                                const int32_t *new_lens,
                                const int32_t *block_table, int32_t max_blocks_per_seq,
                                int32_t block_tokens, int64_t num_phys_blocks,
                                const int32_t *kt_block_table, int32_t kt_max_blocks_per_seq,
                                int32_t kt_block_tokens, int64_t num_kt_blocks,
                                int32_t batch, int32_t max_new, int32_t heads, int32_t head_dim,
                                int32_t *status_flags, void *cuda_stream);

/*
 * Algorithm 1 per (sequence, head), S = seq_lens[b]:
 *   1     I = the r dims of largest |q_d| (ties: lower d)
 *   2-4   approximate weights s^ = softmax_i(q_I . K^T[I, i] * scale / sqrt(|q_I|_1 / |q|_1)),
 *         read from kt_pool (scale = 1/sqrt(head_dim) gives the printed temperature)
 *   5-6   J = the k positions of largest s^, the last `local_window` positions always kept
 *         (ties: lower position); k = k_tokens[b] clipped to S, local_window clipped to k
 *   7     alpha = sum of s^ over J
 *   8-10  exact softmax over J of scale * q . K[j]
 *   11    out = alpha * (weights . V[J]) + (1 - alpha) * v_sum / S
 * The page-then-filter loading of steps 2-3 and 8-9 is a property of flash pages; here rows
 * are gathered directly, which gives the same values.
 *   out       fp16 [batch, heads, head_dim]
 *   alpha     fp32 [batch, heads], nullable
 *   selected  int32 [batch, heads, max_k], nullable: J in ascending order, -1 padded
 *   k_tokens  int32 [batch], device; max_k is a host upper bound (1 <= max_k <= max_seq_len);
 *             a larger k_tokens[b] is clipped to max_k
 *   r         1 <= r <= head_dim
 *   workspace at least instinfer_sparf_workspace_bytes(batch, heads, head_dim, max_seq_len, max_k)
 * Scores and the selection are computed in fp32; two scores closer than fp32 rounding may be
 * ordered differently than in exact arithmetic.  num_phys_blocks * heads * block_tokens must
 * be below 2^31.  S == 0 gives a zero row.
 */
int instinfer_sparf_decode_attention(void *out, float *alpha, int32_t *selected, const void *q,
                                     const void *k_pool, const void *v_pool, const void *kt_pool,
                                     const float *v_sum, const int32_t *block_table,
                                     const int32_t *seq_lens, const int32_t *k_tokens,
                                     int32_t batch, int32_t heads, int32_t head_dim,
                                     int32_t block_tokens, int32_t max_blocks_per_seq,
                                     int64_t num_phys_blocks,
                                     const int32_t *kt_block_table, int32_t kt_max_blocks_per_seq,
                                     int32_t kt_block_tokens, int64_t num_kt_blocks,
                                     int32_t max_seq_len, int32_t max_k,
                                     int32_t r, int32_t local_window, float scale,
                                     void *workspace, size_t workspace_bytes,
                                     int32_t *status_flags, void *cuda_stream);

size_t instinfer_sparf_workspace_bytes(int32_t batch, int32_t heads, int32_t head_dim,
                                       int32_t max_seq_len, int32_t max_k);


/*
 * Workspace size (bytes, host computation only) for a call with these sizes under the
 * current split plan; 0 if an argument is invalid.
 */
size_t instinfer_workspace_bytes(int32_t batch, int32_t heads, int32_t head_dim,
                                 int32_t max_seq_len);

/*
 * Split plan.  A sequence is cut at fixed logical token positions, the same for every
 * sequence: first a few short chunks (they are scheduled last: every sequence of a ragged
 * batch has its first tokens, so every launch ends on short blocks and its tail stays short),
 * then long chunks of `chunk_tokens`.  Each chunk of each (sequence, head) is reduced by one
 * thread block and the partial results are merged by log-sum-exp in position order (no
 * counterpart in the paper, whose engine streams token groups through parallel GeMV units,
 * Sec. IV-B).  instinfer_plan_chunk_tokens returns the long chunk size the library would use
 * for these sizes and instinfer_plan_num_splits the number of chunks per sequence, short ones
 * included (0 if an argument is invalid).
 * instinfer_set_chunk_tokens(n) forces uniform chunks of n tokens for later calls of this
 * process (n > 0, a multiple of 64), n == 0 restores the automatic choice; it returns
 * INSTINFER_OK or INSTINFER_ERR_INVALID_ARG.  Not thread-safe against concurrent calls.
 */
int32_t instinfer_plan_chunk_tokens(int32_t batch, int32_t heads, int32_t max_seq_len);
int32_t instinfer_plan_num_splits(int32_t batch, int32_t heads, int32_t max_seq_len);
/*
 * Small problems (at most 8 chunks of at most 512 tokens per sequence and about two waves of
 * thread blocks in all) are bound by launch and memory latency: there the chunks of one
 * (sequence, head) run as one thread-block cluster, leave their partials in shared memory and
 * are merged inside the same kernel, so the call is one launch instead of two and the
 * workspace is not touched.  Returns 1 if the single-GPU attention entry points would do
 * that for these sizes under the current plan, else 0.
 */
int32_t instinfer_plan_merges_in_cluster(int32_t batch, int32_t heads, int32_t max_seq_len);

/*
 * ======================= Tuning, test and measurement aids =======================
 * The three calls below set process-global state that later calls of the entry points above
 * read.  They exist so that tests can drive every split plan and both forms of the sparse
 * selection, and so that a benchmark can time one kernel where it runs; a serving process
 * never needs them.  None is thread-safe against calls that run at the same time, and none
 * changes a result beyond what its comment says.
 */
int instinfer_set_chunk_tokens(int32_t chunk_tokens);

/*
 * Steps 1-7 of Algorithm 1 have two implementations: one thread block per (sequence, head)
 * that keeps the row's approximate logits in shared memory (rows of at most 16384 tokens), and
 * a chain of kernels for long rows that first brackets the k-th largest score on a sample of
 * the row and then keeps only the tokens that can still be selected (any length; rows it
 * cannot settle, e.g. thousands of equal scores, are redone by one block per row).  Both
 * compute the same fp32 scores and cut ties by position, so they select the same tokens.
 * The library picks by the sizes; instinfer_set_sparse_path forces the choice for later calls
 * of this process: 0 automatic, 1 the chain, 2 one block per row where the rows fit (a tuning
 * and test aid; returns INSTINFER_OK or INSTINFER_ERR_INVALID_ARG; not thread-safe against
 * concurrent calls).
 */
int instinfer_set_sparse_path(int32_t path);

/*
 * instinfer_decode_attention_grouped has two implementations of the same arithmetic: warp-level
 * tensor-core MMAs (every head size and block size the entry point takes) and, for head size
 * 128 or 256 with a contiguous cache or blocks of 16, 32, 64 or a multiple of 128 tokens,
 * asynchronous tcgen05 MMAs that take 128-token tiles as the long side, with accumulators in
 * tensor memory and tiles moved by tensor-map copies.  The library picks the second where the shape allows;
 * instinfer_set_grouped_path forces the choice for later calls of this process: 0 automatic,
 * 1 warp-level, 2 tcgen05 where the shape allows (a tuning and test aid; returns INSTINFER_OK
 * or INSTINFER_ERR_INVALID_ARG; not thread-safe against concurrent calls).  Both meet the
 * entry point's tolerances; their results are not bit-identical to each other.  The setting also
 * holds for instinfer_decode_attention_tree, whose tcgen05 form takes these block sizes and every
 * head size (head size 64 from 17 rows per KV head on).
 */
int instinfer_set_grouped_path(int32_t path);

/*
 * Which of the two implementations instinfer_decode_attention_grouped takes for a head size
 * and a cache layout (block_tokens = 0: contiguous), under the current setting of
 * instinfer_set_grouped_path: 1 warp-level, 2 tcgen05, 0 for a shape the entry point refuses.
 * (A cache of 2^31 rows or more still takes the warp-level form at call time.)  Host only.
 */
int32_t instinfer_grouped_path_for(int32_t head_dim, int32_t block_tokens);


/*
 * Measurement aid (no counterpart in the paper).  Given two cudaEvent_t (as void*, owned by
 * the caller), later attention calls of this process record `before_split` on the stream
 * just before the split-KV kernel and `after_split` just after it, so that the caller can
 * time that one kernel where it runs; (NULL, NULL) switches this off, one NULL is invalid.
 * Each call overwrites the previous recording of the same events.  Not thread-safe.
 */
int instinfer_set_timing_events(void *before_split, void *after_split);

/* Static, human-readable text for a status value (host pointer, never NULL). */
const char *instinfer_status_string(int status);

#ifdef __cplusplus
}
#endif
#endif /* INSTINFER_H_ */
