// Attention of groups of sequences over the paged cache, K and V of the queries' own tokens included: what runs in front of and
// behind the kernel that walks the key tiles (rpx_group_tile.cu), and the float32 form.
//
// For query i of the n of a sequence with len cached tokens, query head h and KV head g = h / group:
//     out = sum_{j <= len - n + i} softmax_j(scale * q . k_j) v_j
// The keys of a group's shared pages and those of the sequence itself are summed apart, each with its own maximum m and sum l,
// and joined: with M = max m,  l = sum l_i 2^(m_i - M),  out = sum o_i 2^(m_i - M) / l.
#include "rpx_group.cuh"

namespace rpx {

namespace group {
rpx_status_t launch_group_tile(const Params& p, int32_t head_dim, const rpx_kv_cache_t& cache, cudaStream_t stream);
}

namespace {

using namespace group;

// ------------------------------------------------------------------ the plan
// One block.  Every sequence gets its entry as if it were alone; groups that share are then given theirs, and their members'
// keys begin behind it.  The first units are a running sum over all entries.
constexpr int kPlanThreads = 1024;

__device__ __forceinline__ Entry make_entry(const Params& p, int32_t tok0, int32_t n, int32_t len, int32_t row, int32_t page0) {
    Entry e = {tok0, n, len, row, page0, 1, 0, 1};
    if (n == 0 || len == 0) {
        e.n = e.len = 0;
        return e;
    }
    e.tiles = len / kTile + (len % kTile != 0 ? 1 : 0);
    // Blocks of at most `cap` rows; of at most 64 where the keys are few, so that probabilities keep their second term: over
    // many keys the rounding averages out.
    const int32_t rows = e.tiles <= 2 && p.cap > 64 ? 64 : p.cap, per = max(1, rows / p.group);
    e.blocks = (n + per - 1) / per;
    // A tile's 64 KB (D = 128) are 1.5 us of this SM's share of HBM once, or the work against a block.
    const int32_t work = 4 + e.block_tokens() * p.group * 12 / 128;
    e.weight = max((15 + e.blocks - 1) / e.blocks, work);
    return e;
}

__global__ void __launch_bounds__(kPlanThreads) group_plan_kernel(const __grid_constant__ Params p) {
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    __shared__ int64_t sums[kPlanThreads / 32];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    for (int32_t s = threadIdx.x; s < p.batch; s += kPlanThreads) {
        Seq q;
        if (!read_seq(p, s, &q)) report(p.status);
        p.entries[p.n_groups + s] = make_entry(p, q.tok0, q.n, q.len, s, 0);
        p.seq_group[s] = -1;
    }
    const bool ascend = groups_ascend(p);  // (a barrier: the entries above are written)
    for (int32_t g = warp; g < p.n_groups; g += kPlanThreads / 32) {
        Group r = {0, 0, 0, 0, -1, 0, 0};
        if (ascend) r = read_group(p, g, lane);
        if (r.shared < 0 && lane == 0) report(p.status);
        const bool shares = r.shared > 0 && r.members > 1;
        if (lane == 0) p.entries[g] = make_entry(p, r.tok0, shares ? r.n : 0, r.shared, r.row, 0);
        if (!shares) continue;
        for (int32_t s = r.first + lane; s < r.last; s += 32) {
            Seq q;
            read_seq(p, s, &q);
            p.entries[p.n_groups + s] = make_entry(p, q.tok0, q.n, q.n > 0 ? q.len - r.shared : 0, s, r.shared / kPage);
            p.seq_group[s] = g;
        }
    }
    __syncthreads();
    const int32_t count = p.n_groups + p.batch;
    int64_t carry = 0;
    for (int32_t base = 0; base < count; base += kPlanThreads) {
        const int32_t e = base + threadIdx.x;
        int64_t x = 0;
        if (e < count) {
            const Entry q = p.entries[e];
            if (q.n > 0) x = q.segment_units() * q.blocks * p.num_kv_heads;
        }
        int64_t sum = x;
#pragma unroll
        for (int off = 1; off < 32; off <<= 1) {
            const int64_t y = __shfl_up_sync(0xffffffffu, sum, off);
            if (lane >= off) sum += y;
        }
        __syncthreads();  // the sums of the round before have been read
        if (lane == 31) sums[warp] = sum;
        __syncthreads();
        int64_t before = carry, total = carry;
        for (int w = 0; w < kPlanThreads / 32; ++w) {
            before += w < warp ? sums[w] : 0;
            total += sums[w];
        }
        if (e < count) p.unit0[e] = before + sum - x;
        carry = total;
    }
    if (threadIdx.x == 0) p.unit0[count] = carry;
}

// ------------------------------------------------------------------ the join
// A warp per row (token, query head) that has more than one set to add up: the shared keys' pieces in order, then its own.
constexpr int kJoinWarps = 8;

template <int D>
__global__ void __launch_bounds__(kJoinWarps * 32) group_join_kernel(const __grid_constant__ Params p) {
    constexpr int kCols = D / 32;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int64_t out_row = static_cast<int64_t>(blockIdx.x) * kJoinWarps + warp, token = out_row / p.num_q_heads;
    if (token >= p.total_tokens) return;  // (never a whole block)
    const int32_t h = static_cast<int32_t>(out_row - token * p.num_q_heads), kv_head = h / p.group, in_group = h - kv_head * p.group;
    Seq seq;
    const int32_t s = find_seq(p, token, lane, &seq);
    asm volatile("griddepcontrol.wait;" ::: "memory");  // (of rows that are left out too: this grid never ends before that one)
    if (s < 0) return;
    const int32_t g = __ldcg(p.seq_group + s), count = p.n_groups + p.batch;
    const int64_t size = piece_units(__ldcg(p.unit0 + count), p.ctas);
    float top = -CUDART_INF_F, sum = 0.f, acc[kCols];
#pragma unroll
    for (int i = 0; i < kCols; ++i) acc[i] = 0.f;
    for (int kind = g < 0 ? 1 : 0; kind < 2; ++kind) {
        const int32_t e = kind == 0 ? g : p.n_groups + s;
        const Entry q = Walk::load(p, e);
        const int32_t in = static_cast<int32_t>(token - q.tok0), per = q.block_tokens(), block = in / per;
        const int32_t row = (in - block * per) * p.group + in_group;
        const int64_t unit = __ldcg(p.unit0 + e) + (static_cast<int64_t>(kv_head) * q.blocks + block) * q.segment_units() + kSegment;
        const int64_t c0 = unit / size;
        const int32_t pieces = static_cast<int32_t>((unit + static_cast<int64_t>(q.tiles - 1) * q.weight) / size - c0) + 1;
        if (pieces == 1 && g < 0) return;  // written whole
#pragma unroll 2
        for (int32_t j = 0; j < pieces; ++j) {
            // a piece keeps the segment it starts in the middle of in its first slot, the one it breaks off in its second
            const int64_t slot = ((c0 + j) * 2 + (j == 0 ? 1 : 0)) * p.cap + row, own_row = kind * p.total_tokens * p.num_q_heads + out_row;
            const float2 ml = pieces == 1 ? __ldcg(p.whole_ml + own_row) : __ldcg(p.part_ml + slot);
            const float* o = (pieces == 1 ? p.whole_o + own_row * D : p.part_o + slot * D) + lane * kCols;
            float v[kCols];
            if constexpr (kCols == 4) *reinterpret_cast<float4*>(v) = __ldcg(reinterpret_cast<const float4*>(o));
            else *reinterpret_cast<float2*>(v) = __ldcg(reinterpret_cast<const float2*>(o));
            if (ml.x == -CUDART_INF_F && ml.y == 0.f) continue;  // no key seen (a NaN sum, of nothing but NaN, goes on)
            const float to = fmaxf(top, ml.x), keep = top == -CUDART_INF_F ? 0.f : fast_exp2(top - to);
            const float f = ml.x == -CUDART_INF_F ? 1.f : fast_exp2(ml.x - to);
            top = to;
            sum = fmaf(sum, keep, f * ml.y);
#pragma unroll
            for (int i = 0; i < kCols; ++i) acc[i] = fmaf(acc[i], keep, f * v[i]);
        }
    }
    const float inv = 1.f / sum;
    uint32_t w[kCols / 2];
#pragma unroll
    for (int i = 0; i < kCols / 2; ++i) w[i] = pack_bf16x2(acc[2 * i] * inv, acc[2 * i + 1] * inv);
    uint32_t* dst = reinterpret_cast<uint32_t*>(static_cast<__nv_bfloat16*>(p.out) + out_row * D + lane * kCols);
    if constexpr (kCols == 4) *reinterpret_cast<uint2*>(dst) = make_uint2(w[0], w[1]);
    else *dst = w[0];
    if (lane == 0 && p.lse != nullptr) p.lse[out_row] = (top + log2f(sum)) * kLn2;
}

// ------------------------------------------------------------------ float32
// For checking: a warp per (token, head); four keys a step, eight lanes to a key with D / 8 of its elements each, and a running
// maximum and sum for each of the four, joined at the end of the row.  Bound by that walk.
constexpr int kRowWarps = 4;

template <int D>
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
    const float* src = static_cast<const float*>(p.q) + token * p.q_stride + static_cast<int64_t>(head) * D + part * U;
#pragma unroll
    for (int u = 0; u < U; ++u) {
        q[u] = __ldg(src + u) * p.scale_log2;
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
    float* dst = static_cast<float*>(p.out) + row * D + part * U;
#pragma unroll
    for (int u = 0; u < U; ++u) {
        acc[u] *= f;
#pragma unroll
        for (int off = 8; off < 32; off <<= 1) acc[u] += __shfl_xor_sync(0xffffffffu, acc[u], off);
        if (sub == 0) dst[u] = acc[u] / l;
    }
    if (p.lse != nullptr && lane == 0) p.lse[row] = (top + log2f(l)) * kLn2;
}

int32_t rows_cap(int64_t rows, int32_t group) {
    const int64_t most = rows > group ? rows : group;
    return most <= 16 ? 16 : most <= 32 ? 32 : most <= 64 ? 64 : 128;
}
int32_t cap_of(int32_t max_q, int32_t max_group, int32_t n_groups, int32_t group) {
    const int32_t most = n_groups > 0 && max_group > max_q ? max_group : max_q;
    return rows_cap(static_cast<int64_t>(most) * group, group);
}
constexpr int kMaxCtas = 148;

// Carves the workspace (NULL: only measures it).
size_t carve(Params& p, int64_t tokens, int32_t entries, int32_t batch, int32_t cap, int32_t heads, int32_t head_dim, void* workspace) {
    uint8_t* ws = static_cast<uint8_t*>(workspace);
    size_t at = 0;
    auto take = [&](size_t bytes) {
        uint8_t* r = ws + at;
        at += align_up(bytes, 256);
        return r;
    };
    const size_t rows = static_cast<size_t>(tokens) * heads * 2, slots = static_cast<size_t>(kMaxCtas) * 2 * cap;
    p.entries = reinterpret_cast<Entry*>(take(static_cast<size_t>(entries) * sizeof(Entry)));
    p.unit0 = reinterpret_cast<int64_t*>(take((static_cast<size_t>(entries) + 1) * sizeof(int64_t)));
    p.seq_group = reinterpret_cast<int32_t*>(take(static_cast<size_t>(batch) * sizeof(int32_t)));
    p.whole_ml = reinterpret_cast<float2*>(take(rows * sizeof(float2)));
    p.part_ml = reinterpret_cast<float2*>(take(slots * sizeof(float2)));
    p.whole_o = reinterpret_cast<float*>(take(rows * head_dim * sizeof(float)));
    p.part_o = reinterpret_cast<float*>(take(slots * head_dim * sizeof(float)));
    return at;
}

}  // namespace

size_t group_workspace(const rpx_attn_desc_t* d, int64_t tokens, int32_t batch, int32_t n_groups, int32_t max_q, int32_t max_group) {
    if (d->dtype == RPX_F32 || batch > INT32_MAX - n_groups - 1) return 0;
    Params p = {};
    return carve(p, tokens, n_groups + batch, batch, cap_of(max_q, max_group, n_groups, d->num_q_heads / d->num_kv_heads), d->num_q_heads, d->head_dim, nullptr);
}

bool group_too_large(const GroupArgs& a) {
    if ((a.total_tokens * a.num_q_heads + kRowWarps - 1) / kRowWarps > INT32_MAX) return true;
    return a.batch > INT32_MAX - a.n_groups - 1 || a.cache->num_blocks * a.num_kv_heads > INT32_MAX / 2;
}

rpx_status_t launch_group_attn(const GroupArgs& a) {
    Params p = make_params(a);
    const int64_t rows = a.total_tokens * a.num_q_heads;
    if (a.dtype == RPX_F32) {
        const unsigned blocks = static_cast<unsigned>((rows + kRowWarps - 1) / kRowWarps);
        if (a.head_dim == 128) group_rows_kernel<128><<<blocks, kRowWarps * 32, 0, a.stream>>>(p);
        else group_rows_kernel<64><<<blocks, kRowWarps * 32, 0, a.stream>>>(p);
        return cudaGetLastError() == cudaSuccess ? RPX_OK : RPX_ERR_CUDA;
    }
    const int sms = sm_count();
    if (sms <= 0) return RPX_ERR_CUDA;
    p.cap = cap_of(a.max_q, a.max_group, a.n_groups, p.group);
    // (without the SM budget: where the line of tiles is cut decides the order of the sums)
    p.ctas = sms < kMaxCtas ? sms : kMaxCtas;
    carve(p, a.total_tokens, a.n_groups + a.batch, a.batch, p.cap, a.num_q_heads, a.head_dim, a.workspace);
    group_plan_kernel<<<1, kPlanThreads, 0, a.stream>>>(p);
    if (cudaGetLastError() != cudaSuccess) return RPX_ERR_CUDA;
    if (rpx_status_t rc = launch_group_tile(p, a.head_dim, *a.cache, a.stream)) return rc;
    const unsigned blocks = static_cast<unsigned>((rows + kJoinWarps - 1) / kJoinWarps);
    return a.head_dim == 128 ? launch_on_top(group_join_kernel<128>, blocks, kJoinWarps * 32, 0, a.stream, p)
                             : launch_on_top(group_join_kernel<64>, blocks, kJoinWarps * 32, 0, a.stream, p);
}

}  // namespace rpx
