// Attention of groups of sequences over the paged cache, K and V of the queries' own tokens included.
//
// For query i of the n of a sequence with len cached tokens, query head h and KV head g = h / group:
//     out = sum_{j <= len - n + i} softmax_j(scale * q . k_j) v_j
//
// This first form takes a warp per (token, head): four keys a step, eight lanes to a key with head_dim / 8 of its elements
// each, and a running maximum and sum for each of the four; they are joined at the end of the row.
#include <cuda_bf16.h>
#include <math_constants.h>

#include "rpx_internal.h"
#include "rpx_ptx.cuh"

namespace rpx {

namespace {

constexpr int kPage = 16;
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

struct Params {
    const void* q;
    int64_t q_stride;
    const int32_t *cu, *lens;
    int32_t batch;
    int64_t total_tokens;
    int32_t max_q, max_group;
    const int32_t *cu_groups, *shared;
    int32_t n_groups;
    int32_t num_q_heads, num_kv_heads, group;
    const int32_t* block_table;
    int32_t block_table_stride, num_blocks;
    const __nv_bfloat16 *k_cache, *v_cache;
    float scale_log2;
    void* out;
    float* lse;
    int32_t* status;
};

__device__ __forceinline__ void report(int32_t* status) {
    if (status != nullptr) atomicCAS(status, 0, RPX_ERR_DEVICE_DATA);
}

// A sequence's queries and cached tokens; false where they do not fit (its rows are left as they are).
struct Seq {
    int32_t tok0, n, len;
};
__device__ __forceinline__ bool read_seq(const Params& p, int32_t s, Seq* q) {
    const int32_t begin = __ldg(p.cu + s), end = __ldg(p.cu + s + 1);
    q->tok0 = begin;
    q->n = 0;
    q->len = 0;
    if (begin < 0 || end < begin || end > p.total_tokens) return false;
    if (end == begin) return true;
    q->len = __ldg(p.lens + s);
    if (end - begin > p.max_q || q->len < end - begin || (static_cast<int64_t>(q->len) + kPage - 1) / kPage > p.block_table_stride) return false;
    q->n = end - begin;
    return true;
}

// The sequence that a token is in, or -1: the last that starts at or before it, 32 offsets a step (a warp together).
__device__ __forceinline__ int32_t find_seq(const Params& p, int64_t token, int lane, Seq* q) {
    int32_t lo = 0, hi = p.batch;
    while (hi - lo > 1) {
        const int32_t step = (hi - lo + 31) / 32;
        const int64_t at = lo + static_cast<int64_t>(lane) * step;
        const uint32_t before = __ballot_sync(0xffffffffu, at < hi && __ldg(p.cu + at) <= token);
        lo += (before != 0u ? 31 - __clz(static_cast<int>(before)) : 0) * step;
        hi = hi - lo > step ? lo + step : hi;
    }
    return read_seq(p, lo, q) && token >= q->tok0 && token < static_cast<int64_t>(q->tok0) + q->n ? lo : -1;
}

// Whether the bounds of all groups ascend (otherwise nothing is shared); by a whole block, which meets at a barrier here.
__device__ __forceinline__ bool groups_ascend(const Params& p) {
    bool good = true;
    for (int32_t g = threadIdx.x; g < p.n_groups; g += blockDim.x) good &= __ldg(p.cu_groups + g) <= __ldg(p.cu_groups + g + 1);
    return __syncthreads_and(good) != 0;
}

// What a group shares: whole pages' tokens, 0 where it has nothing to share, -1 where it does not fit; its first and last
// sequence and their query tokens.  A warp together.
struct Group {
    int32_t first, last, tok0, n, shared;
};
__device__ __forceinline__ Group read_group(const Params& p, int32_t g, int lane) {
    Group r = {__ldg(p.cu_groups + g), __ldg(p.cu_groups + g + 1), 0, 0, -1};
    const int32_t shared = __ldg(p.shared + g);
    if (r.first < 0 || r.last < r.first || r.last > p.batch) return r;
    if (shared < 0) return r;
    bool fits = true;
    for (int32_t s = r.first + lane; s < r.last; s += 32) {
        Seq q;
        fits &= read_seq(p, s, &q) && (q.n == 0 || q.len - q.n >= shared);
    }
    if (!__all_sync(0xffffffffu, fits)) return r;
    if (r.first < r.last) {
        r.tok0 = __ldg(p.cu + r.first);
        r.n = __ldg(p.cu + r.last) - r.tok0;
    }
    if (r.n > p.max_group) return r;
    r.shared = shared / kPage * kPage;
    return r;
}

constexpr int kRowWarps = 4;

__device__ __forceinline__ float load_q(const float* p) { return __ldg(p); }
__device__ __forceinline__ float load_q(const __nv_bfloat16* p) { return __bfloat162float(*p); }
__device__ __forceinline__ void store_out(float* p, float x) { *p = x; }
__device__ __forceinline__ void store_out(__nv_bfloat16* p, float x) { *p = __float2bfloat16_rn(x); }

template <class T, int D>
__global__ void __launch_bounds__(kRowWarps * 32) group_rows_kernel(const Params p) {
    constexpr int U = D / 8;  // elements of a lane
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, sub = lane >> 3, part = lane & 7;
    if (blockIdx.x == 0) {  // what does not fit is reported once
        Seq q;
        for (int32_t s = threadIdx.x; s < p.batch; s += blockDim.x)
            if (!read_seq(p, s, &q)) report(p.status);
        const bool ascend = groups_ascend(p);
        for (int32_t g = warp; g < p.n_groups; g += kRowWarps)
            if (!ascend || read_group(p, g, lane).shared < 0) report(p.status);
    }
    const int64_t row = static_cast<int64_t>(blockIdx.x) * kRowWarps + warp;
    const int64_t token = row / p.num_q_heads;
    const int32_t head = static_cast<int32_t>(row - token * p.num_q_heads);
    if (token >= p.total_tokens) return;
    Seq seq;
    const int32_t s = find_seq(p, token, lane, &seq);
    if (s < 0) return;
    float q[U], acc[U];
    const T* src = static_cast<const T*>(p.q) + token * p.q_stride + static_cast<int64_t>(head) * D + part * U;
#pragma unroll
    for (int u = 0; u < U; ++u) {
        q[u] = load_q(src + u) * p.scale_log2;
        acc[u] = 0.f;
    }
    float m = -CUDART_INF_F, l = 0.f;
    bool bad_page = false;
    const int32_t keys = seq.len - seq.n + static_cast<int32_t>(token - seq.tok0) + 1;
    const int32_t* table = p.block_table + static_cast<int64_t>(s) * p.block_table_stride;
    for (int32_t j0 = 0; j0 < keys; j0 += 4) {
        const int32_t j = j0 + sub;
        const int32_t block = j < keys ? __ldg(table + j / kPage) : 0;
        const bool there = j < keys && block >= 0 && block < p.num_blocks;
        bad_page |= j < keys && !there;
        float x = 0.f;
        uint4 v[U / 8];
        if (there) {
            const int64_t at = ((static_cast<int64_t>(block) * p.num_kv_heads + head / p.group) * kPage + j % kPage) * D + part * U;
#pragma unroll
            for (int c = 0; c < U / 8; ++c) {
                const uint4 k = __ldg(reinterpret_cast<const uint4*>(p.k_cache + at) + c);
                v[c] = __ldg(reinterpret_cast<const uint4*>(p.v_cache + at) + c);
                const uint32_t w[4] = {k.x, k.y, k.z, k.w};
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    x = fmaf(q[8 * c + 2 * i], __uint_as_float(w[i] << 16), x);
                    x = fmaf(q[8 * c + 2 * i + 1], __uint_as_float(w[i] & 0xffff0000u), x);
                }
            }
        }
#pragma unroll
        for (int off = 4; off > 0; off >>= 1) x += __shfl_xor_sync(0xffffffffu, x, off);
        if (!there) continue;
        const float to = fmaxf(m, x);
        const float base = to == -CUDART_INF_F ? 0.f : to;  // nothing but scores of -inf so far
        const float keep = exp2f(m - base), e = exp2f(x - base);
        l = fmaf(l, keep, e);
        m = to;
#pragma unroll
        for (int c = 0; c < U / 8; ++c) {
            const uint32_t w[4] = {v[c].x, v[c].y, v[c].z, v[c].w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                acc[8 * c + 2 * i] = fmaf(acc[8 * c + 2 * i], keep, e * __uint_as_float(w[i] << 16));
                acc[8 * c + 2 * i + 1] = fmaf(acc[8 * c + 2 * i + 1], keep, e * __uint_as_float(w[i] & 0xffff0000u));
            }
        }
    }
    if (__any_sync(0xffffffffu, bad_page) && lane == 0) report(p.status);
    // ---- the four quarters of the keys
    float top = m;
#pragma unroll
    for (int off = 8; off < 32; off <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, off));
    const float f = m == -CUDART_INF_F && l == l ? 0.f : exp2f(m - top);  // (a quarter that saw no key; a NaN sum goes on)
    l *= f;
#pragma unroll
    for (int off = 8; off < 32; off <<= 1) l += __shfl_xor_sync(0xffffffffu, l, off);
    T* dst = static_cast<T*>(p.out) + row * D + part * U;
#pragma unroll
    for (int u = 0; u < U; ++u) {
        acc[u] *= f;
#pragma unroll
        for (int off = 8; off < 32; off <<= 1) acc[u] += __shfl_xor_sync(0xffffffffu, acc[u], off);
        if (sub == 0) store_out(dst + u, acc[u] / l);
    }
    if (p.lse != nullptr && lane == 0) p.lse[row] = (top + log2f(l)) * kLn2;
}

template <class T>
rpx_status_t launch_rows(const Params& p, const GroupArgs& a) {
    const int64_t blocks = (a.total_tokens * a.num_q_heads + kRowWarps - 1) / kRowWarps;
    if (a.head_dim == 128) group_rows_kernel<T, 128><<<static_cast<unsigned>(blocks), kRowWarps * 32, 0, a.stream>>>(p);
    else group_rows_kernel<T, 64><<<static_cast<unsigned>(blocks), kRowWarps * 32, 0, a.stream>>>(p);
    return cudaGetLastError() == cudaSuccess ? RPX_OK : RPX_ERR_CUDA;
}

}  // namespace

size_t group_workspace(const rpx_attn_desc_t*, int64_t, int32_t, int32_t, int32_t, int32_t) { return 0; }

bool group_too_large(const GroupArgs& a) { return (a.total_tokens * a.num_q_heads + kRowWarps - 1) / kRowWarps > INT32_MAX; }

rpx_status_t launch_group_attn(const GroupArgs& a) {
    Params p = {};
    p.q = a.q;
    p.q_stride = a.q_tok_stride;
    p.cu = a.cu;
    p.lens = a.kv_lens;
    p.batch = a.batch;
    p.total_tokens = a.total_tokens;
    p.max_q = a.max_q;
    p.max_group = a.max_group;
    p.cu_groups = a.cu_groups;
    p.shared = a.shared_lens;
    p.n_groups = a.n_groups;
    p.num_q_heads = a.num_q_heads;
    p.num_kv_heads = a.num_kv_heads;
    p.group = a.num_q_heads / a.num_kv_heads;
    p.block_table = a.cache->block_table;
    p.block_table_stride = a.cache->block_table_stride;
    p.num_blocks = static_cast<int32_t>(a.cache->num_blocks);
    p.k_cache = static_cast<const __nv_bfloat16*>(a.cache->k_cache);
    p.v_cache = static_cast<const __nv_bfloat16*>(a.cache->v_cache);
    const float scale = a.softmax_scale > 0.f ? a.softmax_scale : 1.0f / sqrtf(static_cast<float>(a.head_dim));
    p.scale_log2 = scale * kLog2e;
    p.out = a.out;
    p.lse = a.lse;
    p.status = a.device_status;
    return a.dtype == RPX_F32 ? launch_rows<float>(p, a) : launch_rows<__nv_bfloat16>(p, a);
}

}  // namespace rpx
