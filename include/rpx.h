/*
 * rpx — prefix/suffix scoring kernels for NVIDIA B200 (sm_100a), C ABI.
 *
 * The operations follow the paper's statement of the problem (Section 2.3 "Observation and
 * Opportunity"; Section 3.1 Phases 1-2; Table 4, rows "Boundary prefix KV" and "Prefix
 * logprobs"): every model invocation of an RL iteration is split at the first response position
 * into a response-independent PREFIX (the prompt: visual + text tokens) and a response SUFFIX.
 * The prefix pass produces boundary KV state and prefix log-probabilities before the responses
 * exist; the suffix pass consumes the responses together with the retained boundary KV; prefix
 * and suffix log-probabilities together are the full-sequence values.
 *
 * Conventions for every entry point
 *   - All tensor pointers are DEVICE pointers unless marked "host".  Descriptor structs
 *     (rpx_attn_desc_t, rpx_kv_cache_t) are read on the HOST during the call.
 *   - The caller owns every buffer (inputs, outputs, cache pool, block table, workspace, status
 *     word) and must keep it alive until `cuda_stream` has executed the enqueued work.  The
 *     library allocates no device memory, keeps no state between calls (but see
 *     rpx_set_sm_budget) and never synchronises: a call only enqueues kernels, and small
 *     asynchronous memsets of its workspace, on `cuda_stream` (a cudaStream_t passed as void*,
 *     NULL = the legacy default stream) of the current device.
 *   - A workspace belongs to one call at a time: the kernels keep their work-item counters and
 *     partial results there, so two calls that may overlap on the GPU (different streams) need
 *     different workspaces.  Calls on one stream may share one.
 *   - Packed layouts: a [tokens][heads][head_dim] tensor has head_dim contiguous, heads
 *     contiguous (stride head_dim) and a caller-given token stride in ELEMENTS.  Sequence s owns
 *     tokens cu_seqlens[s] .. cu_seqlens[s+1]-1 (int32, device, batch+1 entries, cu_seqlens[0]=0).
 *   - Query head h reads KV head h / (num_q_heads / num_kv_heads).
 *   - Element types: RPX_BF16 tensors are bfloat16.  RPX_F32 tensors are float32 and exist for checking the
 *     method against an unrounded reference, not for throughput: the attention calls then run an fp32 CUDA-core
 *     kernel (q, the call's own k, v and every product stay fp32; out is float32), and the LM-head calls round
 *     hidden and w_vocab to bf16 (nearest-even) in a pre-pass into the workspace before the tensor-core kernel.
 *     The KV cache is always bf16: an RPX_F32 prefix pass stores K and V rounded to nearest-even, and a later
 *     suffix or chunk pass reads those rounded values, as the bf16 path does.
 *   - Host-checkable problems (NULL pointer, head counts, head_dim, block size, alignment,
 *     strides, workspace size, device architecture) return a negative status BEFORE any launch.
 *     Problems only visible on the device (a kernel-side wait that ran out, an out-of-range
 *     target id or block id, sequence offsets that run backwards or past the end of the packed
 *     tensors, a sequence with more pages than a row of the block table) are written to *device_status (nullable, device int32, zeroed by the
 *     caller): the first error code wins; the caller reads it after its own synchronisation.
 *     Every kernel-side wait is bounded: on expiry the kernel records RPX_ERR_TIMEOUT, drains and
 *     returns; outputs of that call are then undefined.
 *   - Alignment: every tensor pointer 16-byte aligned; token/row strides multiples of 8 elements;
 *     every workspace pointer 256-byte aligned (RPX_ERR_ALIGN otherwise, before any launch).
 *   - Zero-length sequences, batch == 0 and n_tokens == 0 are legal no-ops.
 */
#ifndef RPX_H_
#define RPX_H_

#include <stddef.h>
#include <stdint.h>

#if defined(__GNUC__)
#define RPX_API __attribute__((visibility("default")))
#else
#define RPX_API
#endif

#ifdef __cplusplus
extern "C" {
#endif

typedef int32_t rpx_status_t;
enum {
    RPX_OK = 0,
    RPX_ERR_NULL = -1,        /* a required pointer is NULL                                  */
    RPX_ERR_SHAPE = -2,       /* unsupported or inconsistent sizes                           */
    RPX_ERR_DTYPE = -3,       /* unknown element type                                        */
    RPX_ERR_ALIGN = -4,       /* pointer or stride alignment                                 */
    RPX_ERR_WORKSPACE = -5,   /* workspace NULL or smaller than *_workspace_bytes            */
    RPX_ERR_ARCH = -6,        /* current device is not compute capability 10.x               */
    RPX_ERR_CUDA = -7,        /* a CUDA runtime/driver call failed                           */
    RPX_ERR_DEVICE_DATA = -8, /* (device_status) out-of-range id found in device data        */
    RPX_ERR_TIMEOUT = -9,     /* (device_status) a bounded kernel-side wait expired          */
    RPX_ERR_NO_PAGES = -10    /* (device_status) the page pool has too few free pages        */
};

typedef enum { RPX_BF16 = 0, RPX_F32 = 1 } rpx_dtype_t;

/* Attention problem shape.  head_dim is 64 or 128; num_q_heads % num_kv_heads == 0.
 * softmax_scale <= 0 selects 1/sqrt(head_dim).  No bias, soft-cap, window or dropout. */
typedef struct {
    int32_t num_q_heads;
    int32_t num_kv_heads;
    int32_t head_dim;
    float softmax_scale;
    rpx_dtype_t dtype; /* element type of q, k, v and out */
} rpx_attn_desc_t;

/* Paged boundary-KV cache (Table 4, "Boundary prefix KV": produced by the prefix pass, kept in
 * HBM by the caller, consumed by the suffix pass).
 *   k_cache, v_cache : bf16 [num_blocks][num_kv_heads][block_size][head_dim], 16-byte aligned
 *   block_table      : device int32 [batch][block_table_stride]; prefix position t of sequence s
 *                      lives in slot  block_table[s][t / block_size] * block_size + t % block_size
 *   block_size       : must be 16 */
typedef struct {
    void* k_cache;
    void* v_cache;
    int64_t num_blocks;
    int32_t block_size;
    const int32_t* block_table;
    int32_t block_table_stride;
} rpx_kv_cache_t;

/*
 * Prefix attention + boundary-KV write (Section 3.1, Phase 1: the prompt is prefilled before any
 * response exists, which leaves behind the KV state at the prompt/response boundary).  For every
 * sequence s, query head h and prompt position i:
 *     out[i,h,:] = sum_{j<=i} softmax_j(scale * q[i,h,:].k[j,g,:]) * v[j,g,:],   g = h / group
 * and, when `cache` is non-NULL, K and V of every prompt token are stored (as bf16) at the
 * token's slot of the paged cache; slots no token maps to are not touched.
 *   q [total_tokens][num_q_heads][head_dim], k, v [total_tokens][num_kv_heads][head_dim]
 *   out [total_tokens][num_q_heads][head_dim] contiguous, element type desc->dtype
 *   lse (nullable) float32 [total_tokens][num_q_heads]: ln sum_j exp(scale * q.k_j)
 *   max_seqlen: an upper bound on the longest sequence (sizes the grid).  A sequence longer than
 *   the bound rounded up to 256 gets RPX_ERR_DEVICE_DATA in *device_status (its rows beyond the
 *   bound are not computed); the same holds for max_suffix_len / max_chunk_len below.
 */
RPX_API rpx_status_t rpx_prefix_attn(const rpx_attn_desc_t* desc, const void* q, const void* k, const void* v,
                             int64_t q_tok_stride, int64_t k_tok_stride, int64_t v_tok_stride,
                             const int32_t* cu_seqlens, int32_t batch, int64_t total_tokens,
                             int32_t max_seqlen, const rpx_kv_cache_t* cache, void* out, float* lse,
                             void* workspace, size_t workspace_bytes, int32_t* device_status,
                             void* cuda_stream);

/*
 * Suffix attention over the retained boundary (Section 3.1, Phase 2: the suffix pass takes the
 * responses together with the boundary state kept from Phase 1; Section 2.3: the prompt is not
 * computed a second time).  Response position r of sequence s (global
 * position prefix_lens[s] + r) attends to all prefix_lens[s] cached keys and to response keys
 * 0..r; the result equals rows prefix_lens[s].. of one-pass attention over the whole sequence.
 *   q, k, v: response tokens only, packed by cu_seqlens_suffix; prefix_lens device int32 [batch]
 *   cache: required, read-only here (response K/V are NOT appended; they have no later reader)
 *   workspace: rpx_suffix_attn_workspace_bytes includes, for passes of up to 113 664 (token, head) rows,
 *   room for split-KV partials: when the batch is a few long items, the cached prefix of each is cut
 *   into ranges worked on by different SMs and merged by the last to finish (same result up to fp32
 *   rounding of the merge, identical from run to run).
 *   max_suffix_len / max_prefix_len: upper bounds (grid sizing only).
 */
RPX_API rpx_status_t rpx_suffix_attn(const rpx_attn_desc_t* desc, const void* q, const void* k, const void* v,
                             int64_t q_tok_stride, int64_t k_tok_stride, int64_t v_tok_stride,
                             const int32_t* cu_seqlens_suffix, const int32_t* prefix_lens, int32_t batch,
                             int64_t total_suffix_tokens, int32_t max_suffix_len, int32_t max_prefix_len,
                             const rpx_kv_cache_t* cache, void* out, float* lse, void* workspace,
                             size_t workspace_bytes, int32_t* device_status, void* cuda_stream);

/*
 * Chunked prefill of the prefix (an extension: the paper prefills each prompt in one pass and only
 * fixes a per-prompt token budget, Section 4.1).  One call handles the next chunk of every prompt:
 * chunk position i of sequence s (global position cached_lens[s] + i) attends to the cached_lens[s]
 * keys already in the cache and to chunk keys 0..i, exactly as rpx_suffix_attn does, AND the
 * chunk's K and V are appended to the cache at global positions cached_lens[s] + i, exactly as
 * rpx_prefix_attn stores them.  After the last chunk the cache and the concatenated outputs equal
 * those of one rpx_prefix_attn call over the whole prompts.
 *   cached_lens device int32 [batch]: tokens already cached; each must be a multiple of the
 *   block size (chunks start on a page edge) — otherwise nothing is stored for that sequence and
 *   RPX_ERR_DEVICE_DATA appears in *device_status (its attention rows are still computed).
 *   The block table must cover cached_lens[s] + chunk length.  A sequence whose chunk is empty
 *   (cu_seqlens_chunk[s] == cu_seqlens_chunk[s+1]) is skipped whatever its cached_lens.
 *   Other arguments as rpx_suffix_attn; workspace as rpx_suffix_attn_workspace_bytes.
 */
RPX_API rpx_status_t rpx_chunk_attn(const rpx_attn_desc_t* desc, const void* q, const void* k, const void* v,
                            int64_t q_tok_stride, int64_t k_tok_stride, int64_t v_tok_stride,
                            const int32_t* cu_seqlens_chunk, const int32_t* cached_lens, int32_t batch,
                            int64_t total_chunk_tokens, int32_t max_chunk_len, int32_t max_cached_len,
                            const rpx_kv_cache_t* cache, void* out, float* lse, void* workspace,
                            size_t workspace_bytes, int32_t* device_status, void* cuda_stream);

/*
 * Attention of a tree of drafted tokens over the cache (an extension: drafting and verifying several continuations of a
 * cached prefix in one pass; a tree of one node is a decoding step).  Sequence s owns tokens cu_seqlens_tree[s] ..
 * cu_seqlens_tree[s+1]-1, its nodes; node i attends to the cached_lens[s] keys in the cache, to its ancestors in the tree
 * and to itself.
 *   parents: device int32 [total_tree_tokens], per node the number WITHIN its sequence of the node it continues
 *       (0 <= parent < i), -1: it continues the cached prefix, below -1: the node is not in use (padding).  A node not in
 *       use has out = 0 and lse = -inf, is nobody's ancestor, and its k, v may hold anything.  A parent that is not an
 *       earlier node in use sets RPX_ERR_DEVICE_DATA in *device_status; that node and those behind it count as not in use.
 *   cached_lens device int32 [batch]: any length, 0 included.  Slots of the cache behind it may hold anything.
 *   q, k, v, strides, out, lse, cache: as in rpx_suffix_attn.  The tree's K, V are not stored: rpx_cache_append stores
 *       those of the accepted path.  Values of nodes in use are finite: a non-finite one reaches all rows of its sequence.
 *   max_tree_len: upper bound of a sequence's nodes, at most RPX_TREE_MAX_NODES; a longer sequence is reported
 *       (RPX_ERR_DEVICE_DATA) and skipped, as is one whose offsets leave the packed tensors or the block table.
 *   max_cached_len: upper bound of cached_lens (sizes the grid only)
 *   num_q_heads / num_kv_heads: any up to 128; above, RPX_BF16 trees have at most 128 nodes (RPX_ERR_SHAPE)
 *   workspace: rpx_tree_attn_workspace_bytes with the same total_tree_tokens, batch and max_tree_len
 * Results do not depend on the order in which the GPU runs the pieces: the same call gives the same bits.  (Where sequences are
 * cut into pieces goes by all lengths of the batch, so a sequence's sums may round otherwise beside other sequences.)
 * RPX_BF16 calls are not capped by rpx_set_sm_budget; their scores, maxima, sums and outputs are float32 until the output's
 * rounding.  Probabilities enter the product with V as two bf16 terms (off by 2^-17) while a tree has at most 32 rows of
 * nodes times heads of a KV head, or a sequence at most 128 cached keys and 128 nodes; else as one, off by up to 2^-8 each,
 * which averages out over the keys: 0.0023 of the largest output in the worst case measured, against 0.0017 for the output's
 * own rounding.
 */
#define RPX_TREE_MAX_NODES 1024
RPX_API rpx_status_t rpx_tree_attn(const rpx_attn_desc_t* desc, const void* q, const void* k, const void* v,
                                   int64_t q_tok_stride, int64_t k_tok_stride, int64_t v_tok_stride,
                                   const int32_t* cu_seqlens_tree, const int32_t* parents, const int32_t* cached_lens,
                                   int32_t batch, int64_t total_tree_tokens, int32_t max_tree_len, int32_t max_cached_len,
                                   const rpx_kv_cache_t* cache, void* out, float* lse, void* workspace,
                                   size_t workspace_bytes, int32_t* device_status, void* cuda_stream);
RPX_API size_t rpx_tree_attn_workspace_bytes(const rpx_attn_desc_t* desc, int64_t total_tree_tokens, int32_t batch,
                                             int32_t max_tree_len);

/*
 * Fused LM-head log-probabilities (Section 3.1: Phase 1 yields the log-probabilities of the prefix
 * positions, Phase 2 those of the suffix; Table 4, row on prefix log-probabilities).  For every row n:
 *     z_v = hidden[n,:] . w_vocab[v,:]          (never stored)
 *     logprobs[n] = z_{target_ids[n]} - ln sum_v exp(z_v)
 *   hidden [n_tokens][hidden_dim] with row stride in elements; w_vocab [vocab][hidden_dim]
 *   row-major contiguous; target_ids device int32 [n_tokens]; hidden_dim % 8 == 0.
 *   logprobs float32 [n_tokens]; lse (nullable) float32 [n_tokens].
 * A target outside [0, vocab) gives NaN for that row and RPX_ERR_DEVICE_DATA in *device_status.
 * The kernel is position-agnostic: which (hidden row, next token) pairs form the prefix call and
 * which the suffix call is the caller's choice.
 */
RPX_API rpx_status_t rpx_token_logprobs(const void* hidden, int64_t hidden_row_stride, const void* w_vocab,
                                const int32_t* target_ids, int64_t n_tokens, int32_t hidden_dim,
                                int32_t vocab, rpx_dtype_t dtype, float* logprobs, float* lse,
                                void* workspace, size_t workspace_bytes, int32_t* device_status,
                                void* cuda_stream);

/*
 * rpx_token_logprobs with one more output from the same pass (an extension; the paper only needs
 * the log-probs): entropy[n] = - sum_v p_v ln p_v of the next-token distribution p = softmax(z[n,:]),
 * float32 [n_tokens], nullable.  It costs one more multiply-add per logit in the epilogue and no
 * extra memory traffic; every other argument, the workspace size and the error behaviour are those
 * of rpx_token_logprobs (which is this call with entropy == NULL).
 */
RPX_API rpx_status_t rpx_token_logprobs_entropy(const void* hidden, int64_t hidden_row_stride, const void* w_vocab,
                                                const int32_t* target_ids, int64_t n_tokens, int32_t hidden_dim,
                                                int32_t vocab, rpx_dtype_t dtype, float* logprobs, float* lse,
                                                float* entropy, void* workspace, size_t workspace_bytes,
                                                int32_t* device_status, void* cuda_stream);

/*
 * Vocabulary-parallel LM head (an extension; it is how a tensor-parallel reference model, such as
 * the paper's TP=8 one, lays out its LM head).  Each rank holds the rows vocab_begin ..
 * vocab_begin + vocab_local - 1 of W_vocab and calls rpx_token_logprobs_shard on the full hidden
 * rows; the call leaves one 16-byte record per row in shard_stats (float [n_tokens][4], 16-byte
 * aligned): (running max in log2 units, sum of 2^(x - max), target logit if the target lies in
 * this shard else 0, sum of 2^(x - max) * logit).  The ranks exchange their records (one
 * all-gather of 16 bytes per row and rank) and every rank calls rpx_token_logprobs_merge on the
 * gathered array float [n_shards][n_tokens][4]; the result equals rpx_token_logprobs(_entropy) on
 * the whole vocabulary up to fp32 summation order.  target_ids hold GLOBAL vocabulary ids in both
 * calls; workspace as rpx_token_logprobs_workspace_bytes(n_tokens, hidden_dim, vocab_local, dtype).
 */
RPX_API rpx_status_t rpx_token_logprobs_shard(const void* hidden, int64_t hidden_row_stride, const void* w_shard,
                                              const int32_t* target_ids, int64_t n_tokens, int32_t hidden_dim,
                                              int32_t vocab_local, int32_t vocab_begin, rpx_dtype_t dtype,
                                              float* shard_stats, void* workspace, size_t workspace_bytes,
                                              int32_t* device_status, void* cuda_stream);
RPX_API rpx_status_t rpx_token_logprobs_merge(const float* shard_stats, int32_t n_shards, const int32_t* target_ids,
                                              int64_t n_tokens, int32_t vocab_total, float* logprobs, float* lse,
                                              float* entropy, int32_t* device_status, void* cuda_stream);

/*
 * Backward of rpx_token_logprobs with respect to the hidden states (Section 3.2, the autograd contract of the
 * training actor: its suffix and prefix passes are differentiated, and the gradient reaches the prefix through
 * the retained boundary; Table 4, the row on the training actor's boundary KV, which stays attached).  The LM head is
 * where that gradient starts.  With p = softmax(z[n,:]), z = hidden . w_vocab^T, and the caller's upstream gradient
 * g[n] = dL / d logprobs[n]:
 *     dL/dz[n,v]   = g[n] * ([v == target_ids[n]] - p_v)           (recomputed from lse, one block of rows at a time)
 *     dhidden[n,:] = sum_v dL/dz[n,v] * w_vocab[v,:]
 *   hidden, w_vocab, target_ids: as in the forward call; bf16 only (RPX_F32 returns RPX_ERR_DTYPE)
 *   lse      device float32 [n_tokens]: the forward call's lse output for the same rows
 *   upstream device float32 [n_tokens]
 *   dhidden  bf16 [n_tokens][hidden_dim] contiguous, 16-byte aligned
 *   workspace: rpx_token_logprobs_backward_workspace_bytes; it holds dL/dz of one block of at most 9472 rows as
 *   bf16 (9472 x 152064 x 2 bytes = 2.9 GB for the 152064-column vocabulary), never of the whole batch.
 * A target outside [0, vocab) contributes no one-hot term and sets RPX_ERR_DEVICE_DATA in *device_status.
 *
 * rpx_token_logprobs_backward_full also produces the weight gradient from the same block-wise dL/dz:
 *     dw[v,:] = sum_n dL/dz[n,v] * hidden[n,:]
 *   dhidden  as above, or NULL to skip it
 *   dw       device float32 [vocab][hidden_dim] contiguous, 16-byte aligned, or NULL to skip it (at least one of the
 *            two must be given); accumulate_dw == 0: written, != 0: the call's gradient is ADDED to what dw holds
 *            (gradient accumulation over micro-batches)
 * The contraction runs over the rows, so both operands are read as MN-major tiles straight from the row-major dL/dz
 * block and hidden tensor.  rpx_token_logprobs_backward is the same call with dw == NULL.
 */
RPX_API rpx_status_t rpx_token_logprobs_backward(const void* hidden, int64_t hidden_row_stride, const void* w_vocab,
                                                 const int32_t* target_ids, const float* lse, const float* upstream,
                                                 int64_t n_tokens, int32_t hidden_dim, int32_t vocab, rpx_dtype_t dtype,
                                                 void* dhidden, void* workspace, size_t workspace_bytes,
                                                 int32_t* device_status, void* cuda_stream);
RPX_API rpx_status_t rpx_token_logprobs_backward_full(const void* hidden, int64_t hidden_row_stride, const void* w_vocab,
                                                      const int32_t* target_ids, const float* lse, const float* upstream,
                                                      int64_t n_tokens, int32_t hidden_dim, int32_t vocab,
                                                      rpx_dtype_t dtype, void* dhidden, float* dw, int32_t accumulate_dw,
                                                      void* workspace, size_t workspace_bytes, int32_t* device_status,
                                                      void* cuda_stream);
RPX_API size_t rpx_token_logprobs_backward_workspace_bytes(int64_t n_tokens, int32_t hidden_dim, int32_t vocab,
                                                           rpx_dtype_t dtype);

/*
 * Clipped policy loss with a KL term, and its gradient (Section 2.1: the log-probabilities of the responses under the policy,
 * the policy that sampled them and the reference enter the loss of the RL step): from rpx_token_logprobs to the `upstream` of
 * rpx_token_logprobs_backward.  Sequence s owns the tokens cu_seqlens[s] .. cu_seqlens[s+1]-1; of them those with mask != 0
 * (mask NULL: all) are counted, n_s of them; what lies at the others is not used.  With l, o, f the three log-probabilities:
 *     d_t = l_t - o_t, or with RPX_RATIO_SEQUENCE its mean over the counted tokens of the sequence;   r_t = exp(d_t)
 *     policy_t = -A r_t,            and where A > 0 and r_t > 1 + clip_high:                 -A (1 + clip_high)
 *                                       where A < 0 and r_t < 1 - clip_low:                  -A (1 - clip_low)
 *                                       where A < 0 and r_t > clip_dual (clip_dual > 0):     -A clip_dual
 *     kl_t = l - f (kl = 1),  (l - f)^2 / 2 (kl = 2),  exp(f - l) - (f - l) - 1 (kl = 3),  0 (kl = 0)
 *     w_t  = 1 / sum of all n_s (RPX_MEAN_TOKENS), or 1 / (n_s * sequences with n_s > 0) (RPX_MEAN_SEQUENCES); with
 *            desc->count > 0 that number in place of the sum, or of the number of sequences (batches in parts)
 *     loss = sum over the counted tokens of w_t (policy_t + kl_coef kl_t)
 *     dlogprobs_t = upstream * w_t (-A r_t where not clipped, else 0, + kl_coef * d kl_t / d l_t);  0 where not counted
 *   logprobs, old_logprobs, ref_logprobs device float32 [n_tokens]; old_logprobs NULL: d = 0 (a step on the policy itself);
 *       ref_logprobs: needed with kl != 0, otherwise not read
 *   advantages device float32: [n_tokens] with desc->adv_per_token, else [batch] (with RPX_RATIO_SEQUENCE always [batch])
 *   mask device uint8 [n_tokens], or NULL.  These arrays may start at any element (16-byte accesses where all allow them).
 *   upstream device float32 [1], the gradient that reaches the loss, or NULL: 1
 *   stats device float32 [6]: loss, sum w policy, sum w kl, sum w [clipped], sum w r, the number of counted tokens
 *   dlogprobs device float32 [n_tokens], or NULL: no gradient; overlaps neither inputs, stats nor workspace (RPX_ERR_SHAPE).
 *       Tokens of no sequence keep what it holds, or with desc->zero_rest get 0 (for a buffer that holds nothing yet: it goes on to
 *       rpx_token_logprobs_backward)
 *   workspace: rpx_policy_loss_workspace_bytes
 * Which side of a border a ratio is on is decided in 64 bits, and all sums (of ratios, policy and KL terms, and the means of d) are
 * in 64 bits, in a fixed order: the same call gives the same bits.  cu_seqlens that do not ascend from 0 or more to n_tokens at
 * most are reported (RPX_ERR_DEVICE_DATA): a sequence that does not fit counts as empty, and the outputs of that call are undefined.
 */
enum { RPX_RATIO_TOKEN = 0, RPX_RATIO_SEQUENCE = 1 };
enum { RPX_MEAN_TOKENS = 0, RPX_MEAN_SEQUENCES = 1 };
typedef struct {
    int32_t ratio;         /* RPX_RATIO_* */
    int32_t mean;          /* RPX_MEAN_* */
    int32_t kl;            /* 0 .. 3 */
    int32_t adv_per_token; /* 0 or 1 */
    double clip_low;       /* 0 <= clip_low < 1: doubles, so that a border is the caller's and not its float32 neighbour */
    double clip_high;      /* >= 0 */
    double clip_dual;      /* 0: off, else > 1 */
    double kl_coef;
    double count;          /* 0: the call's own */
    int32_t zero_rest;     /* not 0: dlogprobs of tokens of no sequence is 0 */
} rpx_policy_desc_t;

RPX_API rpx_status_t rpx_policy_loss(const rpx_policy_desc_t* desc, const float* logprobs, const float* old_logprobs,
                                     const float* ref_logprobs, const float* advantages, const uint8_t* mask,
                                     const int32_t* cu_seqlens, int32_t batch, int64_t n_tokens, const float* upstream,
                                     float* stats, float* dlogprobs, void* workspace, size_t workspace_bytes,
                                     int32_t* device_status, void* cuda_stream);
RPX_API size_t rpx_policy_loss_workspace_bytes(int32_t batch, int64_t n_tokens);

/*
 * Backward of causal GQA attention over packed whole sequences (Section 3.2: the training actor differentiates both
 * its suffix pass and its prefix pass, and the suffix pass's gradient reaches the prompt through the prefix K/V it
 * attended to; Table 4, the row on the boundary KV that stays attached).  A sequence is prompt followed by response;
 * with P the softmax weights of query row (i, h) over the keys j <= i of its sequence (recomputed from lse), g the KV
 * head of h, dP_ij = dout[i,h,:] . v[j,g,:], D_i = sum_c dout[i,h,c] * out[i,h,c] and dS_ij = P_ij (dP_ij - D_i):
 *     dv[j,g,:] = sum_{h in g} sum_{i >= j} P_ij  dout[i,h,:]
 *     dk[j,g,:] = scale * sum_{h in g} sum_{i >= j} dS_ij q[i,h,:]
 *     dq[i,h,:] = scale * sum_{j <= i} dS_ij k[j,g,:]
 *   q, k, v, strides, cu_seqlens, batch, total_tokens, max_seqlen: as in rpx_prefix_attn; bf16 only (RPX_F32
 *       returns RPX_ERR_DTYPE)
 *   out, dout  device bf16 [total_tokens][num_q_heads][head_dim] contiguous: the forward output and its gradient
 *   lse        device float32 [total_tokens][num_q_heads]: the forward pass's lse (natural log)
 *   q_begin, q_end   nullable device int32 [batch]: only the query rows q_begin[s] <= i < q_end[s] of sequence s take
 *       part (clamped to the sequence; NULL = 0 and the sequence length).  Rows outside get dq = 0 and add nothing
 *       to dk, dv.  With q_begin = prompt length the call is the suffix pass's backward (the gradient of the
 *       response rows with respect to their own K/V and to the prompt's K/V); with q_end = prompt length it is
 *       the prefix pass's.
 *   dq         device float32 [total_tokens][num_q_heads][head_dim], written (rows outside the range: 0)
 *   dk, dv     device float32 [total_tokens][num_kv_heads][head_dim]; accumulate_dkv == 0: written;
 *       != 0: the call's dk, dv are ADDED to what the buffers hold, so that the suffix pass's call followed by the
 *       prefix pass's call leaves the same sums as one call over all rows
 *   workspace: rpx_attn_backward_workspace_bytes (D, 4 bytes per token and query head), 256-byte aligned
 * P and dS are rounded to bf16 before they enter the tensor-core products, as P is in the forward pass.
 * cu_seqlens that leave the packed tensors are not followed and set RPX_ERR_DEVICE_DATA in *device_status; so does a
 * sequence longer than max_seqlen rounded up to 128 (its rows beyond the bound take no part).
 */
RPX_API rpx_status_t rpx_attn_backward(const rpx_attn_desc_t* desc, const void* q, const void* k, const void* v,
                                       int64_t q_tok_stride, int64_t k_tok_stride, int64_t v_tok_stride, const void* out,
                                       const void* dout, const float* lse, const int32_t* cu_seqlens,
                                       const int32_t* q_begin, const int32_t* q_end, int32_t batch, int64_t total_tokens,
                                       int32_t max_seqlen, float* dq, float* dk, float* dv, int32_t accumulate_dkv,
                                       void* workspace, size_t workspace_bytes, int32_t* device_status,
                                       void* cuda_stream);
RPX_API size_t rpx_attn_backward_workspace_bytes(const rpx_attn_desc_t* desc, int64_t total_tokens);

/*
 * Pages of the cache, shared and moved on the device (the paper keeps the boundary KV of a prompt for all of its responses,
 * Table 4; these calls keep the books when sequences branch, end and leave holes).  A pool has num_blocks pages; all layers
 * of a model share the books, each with its own k_cache, v_cache.
 *   ref_counts  device int32 [num_blocks]: how many table entries hold the page; 0 = free
 *   block_table device int32 [rows][block_table_stride], of which the first table_cols columns are used: the pages a row
 *               holds, in order from column 0, then -1
 *   lens        device int32 [rows]: cached tokens of the row, at most 16 times its pages
 * Several rows may hold the same page.  All decisions go by numbers (lowest free page first, requests in their order), so
 * the same call leaves the same table.  Calls that touch one pool are issued on one stream, or ordered by the caller.
 */
typedef struct {
    int32_t* block_table;
    int32_t block_table_stride;
    int32_t table_cols;
    int32_t rows;
    int32_t* lens;
    int32_t* ref_counts;
    int32_t num_blocks;
} rpx_page_pool_t;

/*
 * Gives up the pages of `n` rows (device int32 [n]; a row listed twice is given up once): counts go down by one per entry,
 * the entries become -1, lens 0.  A row number outside the table, or an entry nobody was counted for, is reported
 * (RPX_ERR_DEVICE_DATA) and skipped.
 */
RPX_API rpx_status_t rpx_pages_free(const rpx_page_pool_t* pool, const int32_t* rows, int32_t n, int32_t* device_status,
                                    void* cuda_stream);

/*
 * Branches sequences.  Request i (of n; src_rows, dst_rows device int32 [n]), with room for extra_tokens more:
 *   src != dst  row dst, which holds no pages, becomes a branch of row src (-1: of nothing, a new sequence): it shares src's
 *               whole pages (counts go up by one), gets fresh pages from there on up to lens[src] + extra_tokens, and
 *               lens[dst] = lens[src].  If src's last page is partial, (copy_src[i], copy_dst[i]) = (that page, the branch's
 *               own): the caller copies it in every layer (rpx_cache_copy_pages).  Otherwise, and for every refused
 *               request, both are -1.
 *   src == dst  the row keeps its pages and gets fresh ones up to lens + extra_tokens.
 * All rows are read as they were before the call: a row is dst of one request only, and a row that is branched into is no
 * request's src.  Requests that break this, rows outside the table, a dst that holds pages, a src without the last page that
 * its lens counts, or more pages than table_cols are reported (RPX_ERR_DEVICE_DATA) and change nothing.  Any other entry of
 * src that is no page of the pool is reported, copied as it is and not counted.  Fresh pages are taken
 * in the order of the requests; one that needs more than are left, and every later one that needs any, is reported
 * (RPX_ERR_NO_PAGES) and changes nothing.
 *   workspace: rpx_pages_fork_workspace_bytes, 256-byte aligned
 */
RPX_API rpx_status_t rpx_pages_fork(const rpx_page_pool_t* pool, const int32_t* src_rows, const int32_t* dst_rows, int32_t n,
                                    int32_t extra_tokens, int32_t* copy_src, int32_t* copy_dst, void* workspace,
                                    size_t workspace_bytes, int32_t* device_status, void* cuda_stream);
RPX_API size_t rpx_pages_fork_workspace_bytes(const rpx_page_pool_t* pool, int32_t n);

/*
 * Moves the live pages to the low end of the pool: with L of them, the live pages numbered L and above go, in order, to the
 * free numbers below L, and everything from L on is free.  Writes the new table and counts (block_table_out with its own
 * stride, ref_counts_out: the pool's own arrays with their stride, or others that do not overlap them; columns beyond table_cols are not
 * written), the list of moves copy_src, copy_dst (device int32 [num_blocks / 2], -1 behind the last move) for
 * rpx_cache_copy_pages, and L to *n_live (device int32).  pool->lens is not used.  A table entry that names a free page, or
 * none of the pool's, is reported (RPX_ERR_DEVICE_DATA) and becomes -1.
 *   workspace: rpx_pages_compact_workspace_bytes, 256-byte aligned
 */
RPX_API rpx_status_t rpx_pages_compact(const rpx_page_pool_t* pool, int32_t* block_table_out, int32_t block_table_out_stride,
                                       int32_t* ref_counts_out, int32_t* copy_src, int32_t* copy_dst, int32_t* n_live,
                                       void* workspace, size_t workspace_bytes, int32_t* device_status, void* cuda_stream);
RPX_API size_t rpx_pages_compact_workspace_bytes(const rpx_page_pool_t* pool);

/*
 * Copies whole pages within the pools of `layers` layers: page src[i] to page dst[i] of K and of V, i < n (device int32 [n];
 * pairs of -1 are skipped).  No dst may appear twice or be a src of another pair (the lists of the two calls above never do).
 *   k_cache, v_cache: bf16 [layers][num_blocks][num_kv_heads][16][head_dim], layer_stride elements between layers
 *   (a multiple of 8; for one layer any).  Page numbers outside the pool are reported and skipped.
 */
RPX_API rpx_status_t rpx_cache_copy_pages(void* k_cache, void* v_cache, int32_t layers, int64_t layer_stride, int64_t num_blocks,
                                          int32_t num_kv_heads, int32_t head_dim, const int32_t* src, const int32_t* dst,
                                          int64_t n, int32_t* device_status, void* cuda_stream);

/*
 * Stores K and V of chosen tokens behind the cached ones (after rpx_tree_attn: those of the accepted path).  Sequence s
 * gets m = cu_append[s+1] - cu_append[s] tokens at positions cached_lens[s] .. cached_lens[s] + m - 1: the tokens
 * token_ids[cu_append[s] + i] of k and v (device int32 [n_token_ids]), or, with token_ids == NULL, the tokens
 * cu_append[s] + i themselves (n_token_ids is not used then).  cached_lens is not changed.
 *   k, v [total_tokens][num_kv_heads][head_dim], RPX_BF16, or RPX_F32 (rounded to nearest-even as the prefix pass does)
 *   max_append: upper bound of m (a sequence with more is reported and skipped).  Positions need not start a page; slots of
 *   other positions are left as they are.  A sequence whose offsets or table do not fit, and a token or page number out of
 *   range, is reported (RPX_ERR_DEVICE_DATA) and not stored.  Two sequences must not store into the same slot (a page that
 *   rows share is never one that is still filled: rpx_pages_fork gives every branch its own).
 */
RPX_API rpx_status_t rpx_cache_append(const void* k, const void* v, int64_t k_tok_stride, int64_t v_tok_stride,
                                      int64_t total_tokens, int32_t num_kv_heads, int32_t head_dim, rpx_dtype_t dtype,
                                      const int32_t* token_ids, int64_t n_token_ids, const int32_t* cu_append,
                                      const int32_t* cached_lens, int32_t batch, int32_t max_append,
                                      const rpx_kv_cache_t* cache, int32_t* device_status, void* cuda_stream);

/*
 * Attention of groups of sequences that share the pages of a prefix (an extension: the paper's workload samples several
 * responses to every prompt, Section 4.1, and each of them attends to the one boundary KV of the prompt, Table 4).  All K
 * and V lie in the cache, the queries' own among them (rpx_qk_norm_rope_append or rpx_cache_append has stored them): sequence
 * s has kv_lens[s] cached tokens and owns the query tokens cu_seqlens_q[s] .. cu_seqlens_q[s+1]-1, the LAST n of its cached
 * tokens; query i of n attends to the positions 0 .. kv_lens[s] - n + i.  n = 1 everywhere is a decoding step.
 *   q [total_q_tokens][num_q_heads][head_dim], token stride in elements; out, lse as in rpx_suffix_attn; out may be q
 *       itself (contiguous), otherwise it does not overlap q (RPX_ERR_SHAPE)
 *   cu_groups device int32 [n_groups + 1]: group g is the sequences cu_groups[g] .. cu_groups[g+1]-1; every sequence is in
 *       one group (alone, if it shares nothing)
 *   shared_lens device int32 [n_groups]: tokens that the group's sequences have in common from position 0 on.  The table rows
 *       of the group name the same pages for the whole pages among them (as rpx_pages_fork leaves them); those are read once
 *       for the group, through the row of its first sequence with queries.  What is beyond is read through every sequence's own.
 *   A group is computed without sharing, and reported (RPX_ERR_DEVICE_DATA), if its bounds or shared length do not fit: the
 *       shared tokens end in front of every member's first query.  A sequence whose offsets leave the packed tensors or the
 *       table, that has more queries than cached tokens, or more than max_q_len, is reported and its rows are left as they are;
 *       where cu_seqlens_q runs backwards, all rows are.
 *   max_q_len, max_group_tokens: upper bounds of a sequence's and of a group's query tokens (a group with more is computed
 *       without sharing, and reported); max_kv_len: upper bound of kv_lens (>= 0; nothing is
 *       sized by it, the work is laid out from kv_lens themselves)
 *   num_q_heads / num_kv_heads: at most 112 with head_dim 128, 128 with 64 (RPX_ERR_SHAPE); more than 64 go over the keys twice
 *   workspace: rpx_group_attn_workspace_bytes with the same sizes
 * What lies behind kv_lens in a page is not used.  V of a sequence's later query tokens has weight 0 for its earlier ones in the
 * same product: an infinity or NaN there makes those rows NaN too.
 * The same call gives the same bits.  (Where the keys are cut goes by all lengths of the batch, so a sequence's sums may round
 * otherwise beside other sequences.)  RPX_BF16: scores, maxima, sums and outputs are float32 until the output's rounding;
 * probabilities enter the product with V as two bf16 terms (off by 2^-17), whatever the group.  RPX_BF16 calls are not capped by
 * rpx_set_sm_budget: the pieces that the keys are cut into, and with them the order of the sums, are those of a whole GPU.
 * RPX_F32 (for checking; a warp per row, nothing is shared): q, out and all products float32, K and V the cache's bf16.
 */
RPX_API rpx_status_t rpx_group_attn(const rpx_attn_desc_t* desc, const void* q, int64_t q_tok_stride, const int32_t* cu_seqlens_q,
                                    const int32_t* kv_lens, int32_t batch, int64_t total_q_tokens, int32_t max_q_len,
                                    int32_t max_kv_len, const int32_t* cu_groups, const int32_t* shared_lens, int32_t n_groups,
                                    int32_t max_group_tokens, const rpx_kv_cache_t* cache, void* out, float* lse,
                                    void* workspace, size_t workspace_bytes, int32_t* device_status, void* cuda_stream);
RPX_API size_t rpx_group_attn_workspace_bytes(const rpx_attn_desc_t* desc, int64_t total_q_tokens, int32_t batch,
                                              int32_t n_groups, int32_t max_q_len, int32_t max_group_tokens);

/*
 * Norm of queries and keys per head and rotation by position, in one pass (the attention calls of this library take q and
 * k with both already applied; the paper's video prompts are positioned on three axes: time, height, width).  For every
 * token t and head h, with the weight w of that tensor (q_weight or k_weight, [head_dim]):
 *     y = x * (mean(x^2) + eps)^(-1/2) * w                     (y = x when the two weights are NULL)
 *     a_i = positions[pair_axis[i]][t] * inv_freq[i]           for the pairs i < rot_dim / 2
 *     out_i              = y_i cos a_i - y_{i+rot_dim/2} sin a_i
 *     out_{i+rot_dim/2}  = y_{i+rot_dim/2} cos a_i + y_i sin a_i,      out_j = y_j for j >= rot_dim
 * Sums and products are float32, the angles are reduced in 64 bits (any int32 position), and the result is rounded once.
 *   desc->rot_dim: a multiple of 16, 16 .. head_dim; head_dim 64 or 128; any head counts >= 1
 *   desc->pair_axis: HOST array of rot_dim / 2 axis numbers < num_axes (1 .. 8), or NULL: every pair takes axis 0
 *   q [n_tokens][num_q_heads][head_dim], k [n_tokens][num_kv_heads][head_dim] with token strides in elements, such as
 *       views of one fused projection; q_weight, k_weight: element type of q and k, both or neither NULL
 *   positions device int32 [num_axes][pos_axis_stride], pos_axis_stride >= n_tokens, or 0: one row for all axes
 *   inv_freq device float32 [rot_dim / 2]
 *   q_out, k_out with token strides; each may be its input itself (same pointer and stride), otherwise no output
 *       overlaps an input or the other output
 */
typedef struct {
    int32_t num_q_heads;
    int32_t num_kv_heads;
    int32_t head_dim;
    int32_t rot_dim;
    int32_t num_axes;
    const uint8_t* pair_axis; /* host */
    float eps;                /* >= 0 */
    rpx_dtype_t dtype;        /* element type of q, k, the weights and the outputs */
} rpx_rope_desc_t;

RPX_API rpx_status_t rpx_qk_norm_rope(const rpx_rope_desc_t* desc, const void* q, const void* k, int64_t q_tok_stride,
                                      int64_t k_tok_stride, const void* q_weight, const void* k_weight,
                                      const int32_t* positions, int64_t pos_axis_stride, const float* inv_freq,
                                      int64_t n_tokens, void* q_out, void* k_out, int64_t q_out_tok_stride,
                                      int64_t k_out_tok_stride, void* cuda_stream);

/*
 * rpx_qk_norm_rope with K and V stored into the paged cache on the way, for generation steps and prompts: q_out as in
 * rpx_qk_norm_rope; the normed and rotated k and the v of token cu_append[s] + i are stored, as bf16 rounded once, at position
 * cached_lens[s] + i of sequence s (cached_lens is not changed).  The same slots as rpx_cache_append's, without k in between.
 *   q, k, v [n_tokens][heads][head_dim] with token strides, such as views of one fused projection; element type desc->dtype
 *   cu_append device int32 [batch + 1], ascending (where it runs backwards, which is reported, tokens of other sequences may be
 *       left out as well).  Tokens of no sequence are not stored and their q_out is left as it is.
 *   positions as in rpx_qk_norm_rope, or NULL: every axis takes the token's place in its sequence, cached_lens[s] + i
 *   max_append: upper bound of a sequence's tokens.  A sequence with more, or whose offsets or table do not fit, is reported
 *       (RPX_ERR_DEVICE_DATA) and left out, its q_out too; a page number out of the pool is reported and that token's K, V are
 *       not stored.  Two sequences must not store into the same slot.
 */
RPX_API rpx_status_t rpx_qk_norm_rope_append(const rpx_rope_desc_t* desc, const void* q, const void* k, const void* v,
                                             int64_t q_tok_stride, int64_t k_tok_stride, int64_t v_tok_stride,
                                             const void* q_weight, const void* k_weight, const int32_t* positions,
                                             int64_t pos_axis_stride, const float* inv_freq, int64_t n_tokens,
                                             const int32_t* cu_append, const int32_t* cached_lens, int32_t batch,
                                             int32_t max_append, const rpx_kv_cache_t* cache, void* q_out,
                                             int64_t q_out_tok_stride, int32_t* device_status, void* cuda_stream);

/*
 * Backward of rpx_qk_norm_rope (Section 3.2: the training actor's passes are differentiated).  dq, dk are the gradients with
 * respect to its outputs as rpx_attn_backward leaves them: float32, contiguous.  With g = the transposed rotation of the
 * gradient, u = x * (mean(x^2) + eps)^(-1/2) and r that factor:
 *     dw = sum over tokens and heads of g u,      dx = r (g w - u mean(g w u))          (dx = g without weights)
 *   dq_in, dk_in: gradients with respect to q and k, desc->dtype, token strides in elements, no overlap with any input
 *   dq_weight, dk_weight: float32 [head_dim], both or neither NULL, only with weights; accumulate_dw == 0: written,
 *       != 0: added to.  n_tokens == 0 writes zeros (or adds nothing).
 *   workspace: rpx_qk_norm_rope_backward_workspace_bytes, needed when dq_weight and dk_weight are given
 * Sums run in a fixed order: the same call gives the same bits.
 */
RPX_API rpx_status_t rpx_qk_norm_rope_backward(const rpx_rope_desc_t* desc, const void* q, const void* k, int64_t q_tok_stride,
                                               int64_t k_tok_stride, const void* q_weight, const void* k_weight,
                                               const int32_t* positions, int64_t pos_axis_stride, const float* inv_freq,
                                               const float* dq, const float* dk, int64_t n_tokens, void* dq_in, void* dk_in,
                                               int64_t dq_in_tok_stride, int64_t dk_in_tok_stride, float* dq_weight,
                                               float* dk_weight, int32_t accumulate_dw, void* workspace,
                                               size_t workspace_bytes, void* cuda_stream);
RPX_API size_t rpx_qk_norm_rope_backward_workspace_bytes(const rpx_rope_desc_t* desc, int64_t n_tokens);

/*
 * Allocation-free variant of rpx_token_logprobs (the paper has no counterpart: this entry point
 * exists for deployment, not for the method).  It is meant for callers that cannot give the
 * library a workspace because they cannot allocate one: a scoring hook that runs inside an
 * engine which has already handed every free byte of HBM to its KV pool (the co-located
 * rollout/training setting), or a section of a serving loop where calling the device allocator is
 * off limits because cudaMalloc may fail there or stall the whole device while it runs.
 *
 * The per-(vocab chunk, row) partial records that rpx_token_logprobs keeps in the caller's
 * workspace live here in a fixed array of RPX_STATIC_SCRATCH_BYTES inside the library image;
 * every GPU that loads the library holds that array until the process exits.  Inputs and outputs
 * are still the caller's.  bf16 inputs only; the result equals that of rpx_token_logprobs up to the order in
 * which fp32 partial sums are merged (this entry point always cuts the vocabulary into 16-tile chunks, the
 * workspace variant into 2 to 16 tiles depending on the row count).
 *   - Limit: ceil(ceil(vocab / 256) / 16) * n_tokens * 16 bytes must not exceed
 *     RPX_STATIC_SCRATCH_BYTES (vocab 152064 => at most 13797 rows per call); larger problems
 *     return RPX_ERR_WORKSPACE before any launch — split the rows over several calls.
 *   - The first call on each device looks up the array's device address (one host-side runtime
 *     query, no allocation).  Make that first call before starting any stream capture.
 *   - Every call on a device shares the one array, which keeps the previous call's contents.
 *     Nothing in it has to start at zero (each call overwrites every record it later reads), but
 *     two calls that overlap on the GPU (different streams, or different threads) race on it:
 *     issue them on one stream or serialise them yourself.
 *   - No cudaMalloc, cudaFree or allocating library routine is called.
 */
#define RPX_STATIC_SCRATCH_BYTES (8u << 20)
RPX_API rpx_status_t rpx_token_logprobs_static(const void* hidden, int64_t hidden_row_stride, const void* w_vocab,
                                               const int32_t* target_ids, int64_t n_tokens, int32_t hidden_dim,
                                               int32_t vocab, float* logprobs, float* lse, int32_t* device_status,
                                               void* cuda_stream);

/* Workspace sizes in bytes for the calls above (pure host arithmetic; 0 is possible). */
RPX_API size_t rpx_prefix_attn_workspace_bytes(const rpx_attn_desc_t* desc, int64_t total_tokens);
RPX_API size_t rpx_suffix_attn_workspace_bytes(const rpx_attn_desc_t* desc, int64_t total_suffix_tokens);
RPX_API size_t rpx_token_logprobs_workspace_bytes(int64_t n_tokens, int32_t hidden_dim, int32_t vocab,
                                          rpx_dtype_t dtype);

/*
 * Self-test of the bounded kernel-side wait every kernel of this library relies on (no counterpart
 * in the paper).  Enqueues a one-CTA kernel in which one thread waits, for at most `limit_cycles`
 * SM cycles (1 .. 2e9), on a barrier that nothing ever signals; the wait must give up, the kernel
 * must return, and RPX_ERR_TIMEOUT must appear in *device_status (device int32, zeroed by the
 * caller).  The CUDA context stays usable: nothing traps, faults or spins without a limit.
 */
RPX_API rpx_status_t rpx_selftest_bounded_wait(int64_t limit_cycles, int32_t* device_status, void* cuda_stream);

/*
 * SM budget for co-running (Section 3.1, Eq. 1).  The overlap model charges the decode side a
 * slowdown Delta_D for sharing the GPU with prefix work; how large it is depends on how much of
 * the GPU the prefix kernels leave free.  The LM-head and attention kernels are persistent (one
 * CTA per SM, all shared memory of the SM), so left alone they leave nothing.  rpx_set_sm_budget(n)
 * caps their grids at n CTAs for every later call of this process (all devices, all streams; rpx_tree_attn and rpx_group_attn
 * are not capped: a caller who holds SMs back for a co-runner does not run them beside it);
 * 0 removes the cap, n < 0 returns RPX_ERR_SHAPE and changes nothing.  Results do not depend on
 * the budget bit for bit.  Host-only state: no CUDA call, no allocation, nothing set on the GPU.
 */
RPX_API rpx_status_t rpx_set_sm_budget(int32_t sms);
RPX_API int32_t rpx_get_sm_budget(void);

/*
 * Which LM-head kernel later calls of this process use (rpx_token_logprobs, _entropy, _shard, _static): 0 = one
 * CTA per 128 x 256 tile, != 0 = CTA pairs (a cluster of two CTAs per 256 x 256 tile, tcgen05 cta_group::2: each
 * CTA loads its own 128 rows of hidden states and half of the W tile, the even CTA issues the MMAs for both).
 * Results equal each other up to the order of fp32 partial sums (the partial records of a row do not depend on
 * which kernel produced them; the split of the vocabulary into chunks is the same).  Host-only state.
 */
RPX_API rpx_status_t rpx_set_lm_head_pairing(int32_t on);
RPX_API int32_t rpx_get_lm_head_pairing(void);

/* Static string for a status code; never NULL. */
RPX_API const char* rpx_status_string(rpx_status_t status);

/* Library version: major * 10000 + minor * 100 + patch. */
RPX_API int32_t rpx_version(void);

#ifdef __cplusplus
}
#endif
#endif /* RPX_H_ */
