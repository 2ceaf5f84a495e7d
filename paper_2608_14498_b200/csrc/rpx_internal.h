// Host-side declarations shared by the C-ABI front end and the kernel launchers.
#pragma once

#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "rpx.h"

namespace rpx {

// Encodes a tiled bf16 tensor map with 128-byte swizzle (inner box extent must be 64 elements).
// dims/strides innermost first; strides_bytes has rank-1 entries (the innermost is contiguous).
// cuTensorMapEncodeTiled is looked up through the runtime, so libcuda is not a link dependency.
rpx_status_t encode_tmap_bf16(CUtensorMap* map, const void* base, int rank, const uint64_t* dims,
                              const uint64_t* strides_bytes, const uint32_t* box);

int sm_count();                 // multiprocessors of the current device (cached per device)
int sm_budget();                // process-wide cap on persistent grids; 0 = none
void set_sm_budget(int sms);
int lm_head_pairing();          // process-wide: 1 = the LM head runs its CTA-pair (cta_group::2) kernel
void set_lm_head_pairing(int on);
rpx_status_t check_arch();      // RPX_OK on compute capability 10.x

// f32 -> bf16 (round to nearest even) of `rows` rows of `cols` contiguous elements.
rpx_status_t launch_cast_f32_bf16(const float* src, int64_t src_row_stride, __nv_bfloat16_raw* dst, int64_t rows,
                                  int64_t cols, cudaStream_t stream);

struct AttnArgs {
    int32_t num_q_heads, num_kv_heads, head_dim;
    float softmax_scale;
    const void *q, *k, *v;             // bf16
    int64_t q_tok_stride, k_tok_stride, v_tok_stride;
    const int32_t* cu_seqlens;         // query/self-key packing
    const int32_t* prefix_lens;        // NULL for the prefix pass
    int32_t batch;
    int64_t total_tokens;
    int32_t max_q_len, max_prefix_len;
    const rpx_kv_cache_t* cache;       // prefix pass: written (nullable); suffix pass: read
    bool append_cache = false;         // chunked prefill: read the earlier chunks AND append this one
    uint32_t* item_counter = nullptr;  // 4 bytes of workspace: the kernel's work-item counter (zeroed by the launcher)
    void* split_ws = nullptr;          // suffix pass only: room for split-KV partials (attn_split_workspace bytes), or NULL
    // launch_attention_f32 only: a tree of drafted tokens instead of causal rows: ancestor set of every token, tree_words
    // words each (launch_tree_sets)
    const uint32_t* tree_sets = nullptr;
    int32_t tree_words = 0;
    void* out;                         // bf16 (launch_attention) or float32 (launch_attention_f32)
    float* lse;
    int32_t* device_status;
    cudaStream_t stream;
};
rpx_status_t launch_attention(const AttnArgs& a);
// RPX_F32: q, k, v are float32 (strides in elements), out is float32; the cache stays bf16.
rpx_status_t launch_attention_f32(const AttnArgs& a);
// Split-KV workspace of a suffix pass over `tokens` query tokens: arrival counters, (max, sum) pairs and fp32
// partial rows for up to 4 ranges; 0 when the pass is too large to ever be split.
size_t attn_split_workspace(int64_t tokens, int32_t num_q_heads, int32_t head_dim);

struct LogprobArgs {
    const void* hidden;   // bf16 [n][hidden_row_stride]
    int64_t hidden_row_stride;
    const void* w;        // bf16 [vocab][hidden_dim]
    const int32_t* target_ids;
    int64_t n_tokens;
    int32_t hidden_dim, vocab;
    float* logprobs;
    float* lse;
    float* entropy;       // nullable
    void* shard_stats;    // nullable float4 [n_tokens]: emit the merged record instead of final outputs
    int32_t target_offset;  // first vocabulary column of `w` (vocabulary-parallel shards), else 0
    void* partials;       // float4 [logprob_num_chunks(vocab, tiles_per_chunk)][n_tokens]
    int32_t tiles_per_chunk;  // vocabulary tiles (256 columns) one work item sweeps
    int32_t* device_status;
    cudaStream_t stream;
};
int32_t logprob_tiles_per_chunk(int64_t n_tokens, int32_t vocab);  // the default policy
int32_t logprob_num_chunks(int32_t vocab, int32_t tiles_per_chunk);
rpx_status_t launch_token_logprobs(const LogprobArgs& a);
rpx_status_t launch_logprob_merge(const void* shard_stats, int32_t n_shards, const int32_t* target_ids, int64_t n_tokens,
                                  int32_t vocab_total, float* logprobs, float* lse, float* entropy, int32_t* status,
                                  cudaStream_t stream);

struct LogprobBwdArgs {
    const void* hidden;        // bf16 [n][hidden_row_stride]
    int64_t hidden_row_stride;
    const void* w;             // bf16 [vocab][hidden_dim]
    const int32_t* target_ids;
    const float* lse;          // [n], from the forward call
    const float* upstream;     // [n], dL / d logprob
    int64_t n_tokens;
    int32_t hidden_dim, vocab;
    void* dhidden;             // bf16 [n][hidden_dim], nullable
    float* dw = nullptr;       // fp32 [vocab][hidden_dim], nullable
    bool accumulate_dw = false;  // add dW to what the buffer holds
    void* dlogits;             // workspace: bf16 [logprob_backward_block_rows(n)][vocab rounded up to 64]
    int32_t* device_status;
    cudaStream_t stream;
};
int64_t logprob_backward_block_rows(int64_t n_tokens);
size_t logprob_backward_workspace(int64_t n_tokens, int32_t vocab);
rpx_status_t launch_token_logprobs_backward(const LogprobBwdArgs& a);

struct AttnBwdArgs {
    int32_t num_q_heads, num_kv_heads, head_dim;
    float softmax_scale;
    const void *q, *k, *v;      // bf16, packed whole sequences
    int64_t q_tok_stride, k_tok_stride, v_tok_stride;
    const void *out, *dout;     // bf16 [tokens][H_q][d], contiguous
    const float* lse;           // [tokens][H_q]
    const int32_t* cu_seqlens;
    const int32_t *q_begin, *q_end;  // nullable: the query rows of every sequence that take part
    int32_t batch;
    int64_t total_tokens;
    int32_t max_seqlen;
    float *dq, *dk, *dv;        // fp32
    bool accumulate;            // add dK / dV to what the buffers hold
    float* dvec;                // workspace: fp32 [tokens][H_q]
    int32_t* device_status;
    cudaStream_t stream;
};
rpx_status_t launch_attention_backward(const AttnBwdArgs& a);

struct TreeArgs {
    int32_t num_q_heads, num_kv_heads, head_dim;
    float softmax_scale;
    const void *q, *k, *v;
    int64_t q_tok_stride, k_tok_stride, v_tok_stride;
    const int32_t *cu_seqlens, *parents, *cached_lens;
    int32_t batch;
    int64_t total_tokens;
    int32_t max_tree, max_cached;
    const rpx_kv_cache_t* cache;
    void* out;
    float* lse;
    void* workspace;
    int32_t* device_status;
    cudaStream_t stream;
};
bool tree_streams(int32_t max_tree, int32_t group);  // whether the streaming form takes trees of this size
size_t tree_stream_workspace(int32_t batch, int32_t head_dim);
rpx_status_t launch_tree_stream(const TreeArgs& a);  // bf16
size_t tree_tile_workspace(int32_t batch, int32_t head_dim, int32_t max_tree, int32_t group);
// bf16; sets and values as launch_tree_sets leaves them, launched directly before on the same stream
rpx_status_t launch_tree_tile(const TreeArgs& a, const uint32_t* sets, const void* values);
int32_t tree_set_words(int32_t max_tree);            // 32-bit words of one ancestor set, a multiple of 4
// Ancestor sets [tokens][tree_set_words] and, unless NULL, the values with unused rows cleared, bf16
// [tokens + 8 batch][H_kv][d]: token t of sequence s in row t + 8 s.
rpx_status_t launch_tree_sets(const TreeArgs& a, uint32_t* sets, void* v_copy);

struct PageArgs {
    int32_t* block_table;        // [rows][block_table_stride]
    int32_t block_table_stride, table_cols, rows;
    int32_t* lens;               // [rows] cached tokens (free, fork)
    int32_t* ref_counts;         // [num_blocks]
    int32_t num_blocks;
    int32_t* device_status;
    cudaStream_t stream;
};
rpx_status_t launch_pages_free(const PageArgs& a, const int32_t* rows, int32_t n);
size_t pages_fork_workspace(int32_t n, int32_t rows, int32_t num_blocks);
rpx_status_t launch_pages_fork(const PageArgs& a, const int32_t* src_rows, const int32_t* dst_rows, int32_t n, int32_t extra,
                               int32_t* copy_src, int32_t* copy_dst, void* workspace);
size_t pages_compact_workspace(int32_t num_blocks);
rpx_status_t launch_pages_compact(const PageArgs& a, int32_t* table_out, int64_t table_out_stride, int32_t* ref_counts_out,
                                  int32_t* copy_src, int32_t* copy_dst, int32_t* n_live, void* workspace);

struct CopyPagesArgs {
    void *k_cache, *v_cache;
    int64_t layer_stride;        // elements between layers, a multiple of 8
    int32_t layers, num_blocks, num_kv_heads, head_dim;
    const int32_t *src, *dst;    // [n]
    int64_t n;
    int32_t* device_status;
    cudaStream_t stream;
};
rpx_status_t launch_copy_pages(const CopyPagesArgs& a);

struct AppendArgs {
    const void *k, *v;
    int64_t k_tok_stride, v_tok_stride;
    int32_t num_kv_heads, head_dim;
    rpx_dtype_t dtype;
    const int32_t* token_ids;    // nullable
    const int32_t* cu;           // [batch + 1]
    const int32_t* cached_lens;
    int32_t batch, max_append;
    int64_t total_tokens, n_listed;  // tokens of k and v; entries cu may reach (of token_ids, or tokens)
    rpx_kv_cache_t cache;
    int32_t* device_status;
    cudaStream_t stream;
};
rpx_status_t launch_append(const AppendArgs& a);

struct RopeArgs {
    const rpx_rope_desc_t* desc;
    const void *q, *k;
    int64_t q_tok_stride, k_tok_stride;
    const void *q_weight, *k_weight;     // both or neither NULL
    const int32_t* positions;
    int64_t pos_axis_stride;
    const float* inv_freq;
    int64_t n_tokens;
    void *q_out, *k_out;                 // forward: the results; backward: gradients with respect to q and k
    int64_t q_out_tok_stride, k_out_tok_stride;
    const float *dq = nullptr, *dk = nullptr;          // backward only
    float *dq_weight = nullptr, *dk_weight = nullptr;  // backward only, nullable
    bool accumulate_dw = false;
    void* workspace = nullptr;           // backward: one partial row per CTA
    // append only (k_out is not used, positions may be NULL)
    const void* v = nullptr;
    int64_t v_tok_stride = 0;
    const int32_t *cu = nullptr, *cached_lens = nullptr;
    int32_t batch = 0, max_append = 0;
    rpx_kv_cache_t cache = {};
    int32_t* device_status = nullptr;
    cudaStream_t stream;
};
constexpr int kRopeBwdCtasPerSm = 4, kRopeBwdMaxCtas = 1024;
size_t rope_backward_workspace(int32_t head_dim);
rpx_status_t launch_qk_rope(const RopeArgs& a);
rpx_status_t launch_qk_rope_append(const RopeArgs& a);
rpx_status_t launch_qk_rope_backward(const RopeArgs& a);

// Sequences of a call (with its groups) at most: loops over them step by a grid or a block beyond the last one, in 32 bits.
constexpr int32_t kMostSequences = INT32_MAX - 65536;

struct PolicyArgs {
    const rpx_policy_desc_t* desc;
    const float *logprobs, *old_logprobs, *ref_logprobs, *advantages;
    const uint8_t* mask;
    const int32_t* cu;
    int32_t batch;
    int64_t n_tokens;
    const float* upstream;
    float *stats, *dlogprobs;
    void* workspace;
    int32_t* device_status;
    cudaStream_t stream;
};
size_t policy_workspace(int32_t batch, int64_t n_tokens);
rpx_status_t launch_policy_loss(const PolicyArgs& a);

struct GroupArgs {
    int32_t num_q_heads, num_kv_heads, head_dim;
    float softmax_scale;
    rpx_dtype_t dtype;
    const void* q;
    int64_t q_tok_stride;
    const int32_t *cu, *kv_lens;         // [batch + 1], [batch]
    int32_t batch;
    int64_t total_tokens;
    int32_t max_q;
    const int32_t *cu_groups, *shared_lens;  // [n_groups + 1], [n_groups]
    int32_t n_groups, max_group;
    const rpx_kv_cache_t* cache;
    void* out;
    float* lse;
    void* workspace;
    int32_t* device_status;
    cudaStream_t stream;
};
size_t group_workspace(const rpx_attn_desc_t* desc, int64_t total_tokens, int32_t batch, int32_t n_groups, int32_t max_q,
                       int32_t max_group);
int32_t group_most_heads(int32_t head_dim);  // query heads to a KV head that the call takes at most
bool group_too_large(const GroupArgs& a);  // sizes that a launch of the pass cannot hold
rpx_status_t launch_group_attn(const GroupArgs& a);

rpx_status_t launch_bounded_wait_selftest(long long limit_cycles, int32_t* status, cudaStream_t stream);

// Launches a kernel that may start before the one in front of it has ended (it waits by itself where it has to).
template <class Kernel, class... Args>
rpx_status_t launch_on_top(Kernel* kernel, unsigned grid, unsigned threads, size_t smem, cudaStream_t stream, const Args&... args) {
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t config = {};
    config.gridDim = dim3(grid);
    config.blockDim = dim3(threads);
    config.dynamicSmemBytes = smem;
    config.stream = stream;
    config.attrs = attr;
    config.numAttrs = 1;
    return cudaLaunchKernelEx(&config, kernel, args...) == cudaSuccess ? RPX_OK : RPX_ERR_CUDA;
}

inline size_t align_up(size_t x, size_t a) { return (x + a - 1) / a * a; }

}  // namespace rpx
