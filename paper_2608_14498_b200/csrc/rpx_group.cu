// Attention of groups of sequences over the paged cache, K and V of the queries' own tokens included: what runs in front of and
// behind the kernel that walks the key tiles (rpx_group_tile.cu), and the float32 form.
//
// For query i of the n of a sequence with len cached tokens, query head h and KV head g = h / group:
//     out = sum_{j <= len - n + i} softmax_j(scale * q . k_j) v_j
// The keys of a group's shared pages and those of the sequence itself are summed apart, each with its own maximum m and sum l,
// and joined: with M = max m,  l = sum l_i 2^(m_i - M),  out = sum o_i 2^(m_i - M) / l.
#include <algorithm>

#include "rpx_group.cuh"

namespace rpx {

namespace group {
rpx_status_t launch_group_tile(const Params& p, int32_t head_dim, const rpx_kv_cache_t& cache, cudaStream_t stream);
}

namespace {

using namespace group;

// ------------------------------------------------------------------ the plan
// One block, which also finds where every CTA's piece begins.
constexpr int kPlanThreads = 1024;

// Units of the line (20 ns): of a tile's work, rows that add one; and what a segment costs besides: two a row, at most kSegmentWork
// (its rows go out one after the other).
constexpr int kWorkUnits = 48, kRowsAUnit = 8, kSegmentWork = 100;

__device__ __forceinline__ Entry make_entry(const Params& p, int32_t tok0, int32_t n, int32_t len, int32_t row, int32_t page0, int32_t group = -1) {
    Entry e = {tok0, n, len, row, page0, 1, 1, 1, 0, group, len / kTile + (len % kTile != 0 ? 1 : 0)};
    if (n == 0 || len == 0) {
        e.n = e.len = 0;
        return e;
    }
    const int32_t per = p.cap / p.group;  // (at least one token, and no more than Q's box holds)
    e.blocks = n <= per ? 1 : (n + per - 1) / per;
    e.block_tokens = e.blocks == 1 ? n : (n + e.blocks - 1) / e.blocks;
    // A tile's bytes are tile_units of this SM's share of HBM, once for all blocks; the work against a block overlaps with that, what
    // a segment costs besides does not quite.
    const int32_t bytes = p.tile_units / e.blocks, block_rows = e.block_tokens * p.group;
    e.weight = max(bytes, kWorkUnits + block_rows / kRowsAUnit) + min(2 * block_rows, kSegmentWork) / e.tiles;
    return e;
}

__device__ __forceinline__ int64_t entry_units(const Params& p, const Entry& e) { return e.n > 0 ? e.segment_units() * e.blocks * p.num_kv_heads : 0; }

// What the sequences of some groups have in common.
struct GroupBooks {
    int32_t first[kPlanThreads + 1];
    int32_t room[kPlanThreads];     // tokens in front of a member's first query, the least of all members; -1: a member does not fit
    int32_t members[kPlanThreads];  // sequences with queries
    int32_t row[kPlanThreads];      // the first of them
    int32_t shared[kPlanThreads];   // whole pages' tokens; 0: nothing, or nobody to share with
    __device__ __forceinline__ void open(int32_t i, int32_t begin) {
        first[i] = begin;
        room[i] = row[i] = INT32_MAX;
        members[i] = 0;
    }
    __device__ __forceinline__ void add(int32_t i, int32_t s, bool fits, const Seq& q) {
        if (!fits) {
            atomicMin(&room[i], -1);
        } else if (q.n > 0) {
            atomicMin(&room[i], q.len - q.n);
            atomicAdd(&members[i], 1);
            atomicMin(&row[i], s);
        }
    }
    __device__ __forceinline__ int32_t find(int32_t s, int32_t groups) const {  // the last that begins at or before the sequence
        int32_t lo = 0, hi = groups;
        while (hi - lo > 1) {
            const int32_t mid = (lo + hi) / 2;
            if (first[mid] <= s) lo = mid;
            else hi = mid;
        }
        return lo;
    }
};

// The tokens that a group shares: 0 for nothing, or nobody to share with; reports what does not fit.  `first`, `last`: its
// sequences, with their first token and the one behind their last; `ascend` false (some bounds descend): no group fits.
__device__ __forceinline__ bool group_fits(const Params& p, bool ascend, int32_t first, int32_t last, int32_t shared, int32_t room) {
    return ascend && first >= 0 && first <= last && last <= p.batch && shared >= 0 && shared <= room;
}
__device__ __forceinline__ int32_t shared_tokens(const Params& p, bool fits, int32_t n, int32_t shared, int32_t members) {
    fits = fits && n <= p.max_group;
    if (!fits) report(p.status);
    return fits && members > 1 ? shared / kPage * kPage : 0;
}

// Running sum over the block's threads; *total: of all of them.
__device__ __forceinline__ int64_t block_sum(int64_t x, int64_t* sums, int64_t* total) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    int64_t sum = x;
#pragma unroll
    for (int off = 1; off < 32; off <<= 1) {
        const int64_t y = __shfl_up_sync(0xffffffffu, sum, off);
        if (lane >= off) sum += y;
    }
    __syncthreads();  // the sums of the round before have been read
    if (lane == 31) sums[warp] = sum;
    __syncthreads();
    const int64_t w = sums[lane];
    int64_t upto = w;
#pragma unroll
    for (int off = 1; off < 32; off <<= 1) {
        const int64_t y = __shfl_up_sync(0xffffffffu, upto, off);
        if (lane >= off) upto += y;
    }
    *total = __shfl_sync(0xffffffffu, upto, 31);
    return __shfl_sync(0xffffffffu, upto - w, warp) + sum;
}

// The cut, and every CTA's start.
template <class Unit0>
__device__ __forceinline__ void leave_starts(const Params& p, int64_t total, Unit0 unit0) {
    const int32_t i = threadIdx.x;
    if (i >= p.ctas) return;
    const int64_t size = piece_units(total, p.ctas);
    p.starts[i] = find_start(p, total, size, i, unit0);
    if (i == 0) {
        p.cut->size = size;
        p.cut->inverse = 1.0 / static_cast<double>(size);
    }
}

// Up to as many entries as threads: a thread an entry, groups first, everything read once (8 prompts of 8 with 5 tokens
// each: the call takes 53 us, with the form below 55; one prompt of 8: 17.1 and 18.7).
__global__ void __launch_bounds__(kPlanThreads) group_plan_small_kernel(const __grid_constant__ Params p) {
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    __shared__ int64_t sums[kPlanThreads / 32];
    __shared__ int64_t unit0[kPlanThreads];
    __shared__ int32_t cu[kPlanThreads + 1];
    __shared__ GroupBooks books;
    const int32_t g = threadIdx.x, s = g - p.n_groups, count = p.n_groups + p.batch;
    const bool is_group = g < p.n_groups, is_seq = !is_group && g < count;
    int32_t first = 0, last = 0, shared = 0;
    Seq q = {0, 0, 0};
    bool fits = true;
    if (is_group) {
        first = __ldg(p.cu_groups + g);
        last = __ldg(p.cu_groups + g + 1);
        shared = __ldg(p.shared + g);
        books.open(g, first);
        if (g + 1 == p.n_groups) books.first[p.n_groups] = last;
    } else if (is_seq) {
        fits = read_seq(p, s, &q);
        if (!fits) report(p.status);
        cu[s] = q.tok0;
        if (s + 1 == p.batch) cu[p.batch] = __ldg(p.cu + p.batch);
    }
    const bool ascend = __syncthreads_and(!is_group || first <= last) != 0;
    const bool member = is_seq && ascend && p.n_groups > 0 && s >= books.first[0] && s < books.first[p.n_groups];
    const int32_t of = member ? books.find(s, p.n_groups) : -1;
    if (member) books.add(of, s, fits, q);
    // (offsets that run backwards: a row's sequence cannot be looked up, and nothing is computed)
    const bool ordered = __syncthreads_and(!is_seq || cu[s] <= cu[s + 1]) != 0;
    if (!ordered) q.n = 0;
    Entry e = {};
    if (is_group) {
        fits = ordered && group_fits(p, ascend, first, last, shared, books.room[g]);
        const int32_t n = fits ? cu[last] - cu[first] : 0;
        shared = shared_tokens(p, fits, n, shared, books.members[g]);
        books.shared[g] = shared;
        e = make_entry(p, shared > 0 ? cu[first] : 0, shared > 0 ? n : 0, shared, books.row[g], 0);
    }
    __syncthreads();
    if (is_seq) {
        shared = member ? books.shared[of] : 0;
        e = make_entry(p, q.tok0, q.n, q.n > 0 ? q.len - shared : 0, s, shared / kPage, shared > 0 ? of : -1);
    }
    const int64_t units = entry_units(p, e);
    int64_t total;
    e.unit0 = unit0[threadIdx.x] = block_sum(units, sums, &total) - units;
    if (g < count) p.entries[g] = e;
    __syncthreads();
    leave_starts(p, total, [&](int32_t i) { return unit0[i]; });
}

// Any number: every sequence gets its entry as if it were alone; groups that share are then given theirs, kPlanThreads at a time,
// and their members' keys begin behind it.
__global__ void __launch_bounds__(kPlanThreads) group_plan_kernel(const __grid_constant__ Params p) {
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    __shared__ int64_t sums[kPlanThreads / 32];
    __shared__ GroupBooks books;
    bool good = true, in_order = true;
    for (int32_t g = threadIdx.x; g < p.n_groups; g += kPlanThreads) good &= __ldg(p.cu_groups + g) <= __ldg(p.cu_groups + g + 1);
    for (int32_t s = threadIdx.x; s < p.batch; s += kPlanThreads) {
        Seq q;
        if (!read_seq(p, s, &q)) report(p.status);
        p.entries[p.n_groups + s] = make_entry(p, q.tok0, q.n, q.len, s, 0);
        in_order &= __ldg(p.cu + s) <= __ldg(p.cu + s + 1);
    }
    const bool ordered = __syncthreads_and(in_order) != 0, ascend = __syncthreads_and(good) != 0 && ordered;
    if (!ordered)  // (as above)
        for (int32_t s = threadIdx.x; s < p.batch; s += kPlanThreads) p.entries[p.n_groups + s] = make_entry(p, 0, 0, 0, s, 0);
    for (int32_t g0 = 0; g0 < p.n_groups; g0 += kPlanThreads) {
        const int32_t groups = min(kPlanThreads, p.n_groups - g0), g = g0 + threadIdx.x;
        const bool is_group = threadIdx.x < groups;
        if (is_group) books.open(threadIdx.x, __ldg(p.cu_groups + g));
        if (threadIdx.x == 0) books.first[groups] = __ldg(p.cu_groups + g0 + groups);
        __syncthreads();
        // the members of these groups (nobody, where the bounds descend; no bound goes into a sum as it came)
        const int32_t begin = min(max(books.first[0], 0), p.batch), end = ascend ? min(books.first[groups], p.batch) : 0;
        for (int32_t s = begin + threadIdx.x; s < end; s += kPlanThreads) {
            Seq q;
            const bool fits = read_seq(p, s, &q);
            books.add(books.find(s, groups), s, fits, q);
        }
        __syncthreads();
        if (is_group) {
            const int32_t first = books.first[threadIdx.x], last = books.first[threadIdx.x + 1];
            int32_t shared = __ldg(p.shared + g);
            const bool fits = group_fits(p, ascend, first, last, shared, books.room[threadIdx.x]);
            const int32_t tok0 = fits ? __ldg(p.cu + first) : 0, n = fits ? __ldg(p.cu + last) - tok0 : 0;
            shared = shared_tokens(p, fits, n, shared, books.members[threadIdx.x]);
            books.shared[threadIdx.x] = shared;
            p.entries[g] = make_entry(p, tok0, shared > 0 ? n : 0, shared, books.row[threadIdx.x], 0);
        }
        __syncthreads();
        for (int32_t s = begin + threadIdx.x; s < end; s += kPlanThreads) {
            const int32_t i = books.find(s, groups), shared = books.shared[i];
            if (shared == 0) continue;
            Seq q;
            read_seq(p, s, &q);
            p.entries[p.n_groups + s] = make_entry(p, q.tok0, q.n, q.n > 0 ? q.len - shared : 0, s, shared / kPage, g0 + i);
        }
        __syncthreads();
    }
    const int32_t count = p.n_groups + p.batch;
    int64_t carry = 0;
    for (int32_t base = 0; base < count; base += kPlanThreads) {
        const int32_t e = base + threadIdx.x;
        const int64_t x = e < count ? entry_units(p, p.entries[e]) : 0;
        int64_t total;
        const int64_t upto = carry + block_sum(x, sums, &total);
        if (e < count) p.entries[e].unit0 = upto - x;
        carry += total;
    }
    __syncthreads();
    leave_starts(p, carry, [&](int32_t i) { return p.entries[i].unit0; });
}

// ------------------------------------------------------------------ the join
// A warp per row (token, query head), or where there are few rows with many sets, the eight warps of a block: the shared keys'
// pieces in order, then its own, kBatch sets a warp at a time, all of them on their way together (one after the other, 17 sets
// took 6 us).  The code is kept short: at this length a kernel waits for its instructions first; and what all warps read alike -
// the cut, the entries - comes through L1 (10240 warps that asked L2 for the same line waited 3 us for it).
constexpr int kJoinWarps = 8, kBatch = 4;

// The sets of a row against one entry: where the first one lies, how far on the next (twice as far on all others), and how many.
struct Sets {
    int64_t first;
    int32_t step, n;
};
__device__ __forceinline__ Sets find_sets(const Params& p, const Entry& q, int32_t kv_head, int32_t in_group, int32_t in) {
    const int64_t size = p.cut->size;
    const double inverse = p.cut->inverse;
    const int32_t block = q.blocks == 1 ? 0 : in / q.block_tokens;
    const int64_t unit = q.unit0 + (static_cast<int64_t>(kv_head) * q.blocks + block) * q.segment_units() + kSegment;
    const int32_t c0 = piece_of(unit, size, inverse);
    Sets r;
    r.n = piece_of(unit + static_cast<int64_t>(q.tiles - 1) * q.weight, size, inverse) - c0 + 1;
    // a piece keeps the segment it starts in the middle of in its first slot, the one it breaks off in its second
    r.step = p.cap;
    r.first = (static_cast<int64_t>(c0) * 2 + 1) * r.step + (in - block * q.block_tokens) * p.group + in_group;
    return r;
}

template <int D, int kSplit>
__global__ void __launch_bounds__(kJoinWarps * 32, 5) group_join_kernel(const __grid_constant__ Params p) {
    constexpr int kCols = D / 32;
    __shared__ float part_acc[kSplit > 1 ? kSplit : 1][D];
    __shared__ float2 part_ml[kSplit > 1 ? kSplit : 1];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, sub = warp % kSplit;
    const int64_t token = static_cast<int64_t>(blockIdx.x) * (kJoinWarps / kSplit) + warp / kSplit;
    const int32_t in_group = blockIdx.y, kv_head = blockIdx.z;
    const bool there = token < p.total_tokens;
    const int32_t s = last_at_or_before(p.cu, p.batch, there ? token : 0, lane);
    asm volatile("griddepcontrol.wait;" ::: "memory");  // (of rows that are left out too: this grid never ends before that one)
    if (!there) return;
    const Entry own = p.entries[p.n_groups + s];
    if (token < own.tok0 || token - own.tok0 >= own.n) return;  // in no sequence, or in one that does not fit
    const int64_t out_row = token * p.num_q_heads + kv_head * p.step + in_group;
    Sets of_own = find_sets(p, own, kv_head, in_group, static_cast<int32_t>(token - own.tok0)), of_group = {0, 0, 0};
    if (own.group < 0 && of_own.n == 1) return;  // written whole
    if (own.group >= 0) {
        const Entry g = p.entries[own.group];
        of_group = find_sets(p, g, kv_head, in_group, static_cast<int32_t>(token - g.tok0));
    }
    float top = -CUDART_INF_F, sum = 0.f, acc[kCols];
#pragma unroll
    for (int i = 0; i < kCols; ++i) acc[i] = 0.f;
    const int32_t n = of_group.n + of_own.n;
#pragma unroll 1
    for (int32_t j0 = sub; j0 < n; j0 += kSplit * kBatch) {
        float2 ml[kBatch];
        alignas(16) float v[kBatch][kCols];
#pragma unroll
        for (int u = 0; u < kBatch; ++u) {
            const bool shared = j0 + kSplit * u < of_group.n;
            const Sets& of = shared ? of_group : of_own;
            const int32_t j = j0 + kSplit * u - (shared ? 0 : of_group.n);
            int64_t at = of.first + (j == 0 ? 0 : static_cast<int64_t>(2 * j - 1) * of.step);
            const float2* mls = p.part_ml;
            const float* os = p.part_o;
            if (of.n == 1) {  // a segment that is whole: the row's own place
                at = out_row + (shared ? 0 : p.total_tokens * p.num_q_heads);
                mls = p.whole_ml;
                os = p.whole_o;
            }
            ml[u] = make_float2(-CUDART_INF_F, 0.f);
#pragma unroll
            for (int i = 0; i < kCols; ++i) v[u][i] = 0.f;
            if (j0 + kSplit * u < n) {
                ml[u] = __ldcg(mls + at);
                if constexpr (kCols == 4) *reinterpret_cast<float4*>(v[u]) = __ldcg(reinterpret_cast<const float4*>(os + at * D) + lane);
                else *reinterpret_cast<float2*>(v[u]) = __ldcg(reinterpret_cast<const float2*>(os + at * D) + lane);
            }
        }
        float to = top;
#pragma unroll
        for (int u = 0; u < kBatch; ++u) to = fmaxf(to, ml[u].x);
        const float base = to == -CUDART_INF_F ? 0.f : to;  // (no key seen so far)
        const float keep = fast_exp2(top - base);
        top = to;
        sum *= keep;
#pragma unroll
        for (int i = 0; i < kCols; ++i) acc[i] *= keep;
#pragma unroll
        for (int u = 0; u < kBatch; ++u) {
            // a set that saw no key has a sum and outputs of 0; one of nothing but NaN goes on with a factor of 1
            const float f = ml[u].x == -CUDART_INF_F ? 1.f : fast_exp2(ml[u].x - base);
            sum = fmaf(f, ml[u].y, sum);
#pragma unroll
            for (int i = 0; i < kCols; ++i) acc[i] = fmaf(f, v[u][i], acc[i]);
        }
    }
    if constexpr (kSplit > 1) {
#pragma unroll
        for (int i = 0; i < kCols; ++i) part_acc[warp][lane * kCols + i] = acc[i];
        if (lane == 0) part_ml[warp] = make_float2(top, sum);
        __syncthreads();  // (the warps of a block are of one row)
        if (warp != 0) return;
        top = -CUDART_INF_F;
        sum = 0.f;
#pragma unroll
        for (int i = 0; i < kCols; ++i) acc[i] = 0.f;
        for (int w = 0; w < kSplit; ++w) top = fmaxf(top, part_ml[w].x);
        for (int w = 0; w < kSplit; ++w) {
            const float2 ml = part_ml[w];
            const float f = ml.x == -CUDART_INF_F ? 1.f : fast_exp2(ml.x - top);  // (as above)
            sum = fmaf(f, ml.y, sum);
#pragma unroll
            for (int i = 0; i < kCols; ++i) acc[i] = fmaf(f, part_acc[w][lane * kCols + i], acc[i]);
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

template <int D, int kSplit>
rpx_status_t launch_join(const Params& p, cudaStream_t stream) {
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t config = {};
    constexpr int kTokens = kJoinWarps / kSplit;
    config.gridDim = dim3(static_cast<unsigned>((p.total_tokens + kTokens - 1) / kTokens), static_cast<unsigned>(p.group), static_cast<unsigned>(p.num_kv_heads));
    config.blockDim = dim3(kJoinWarps * 32);
    config.stream = stream;
    config.attrs = attr;
    config.numAttrs = 1;
    return cudaLaunchKernelEx(&config, group_join_kernel<D, kSplit>, p) == cudaSuccess ? RPX_OK : RPX_ERR_CUDA;
}
template <int D>
rpx_status_t launch_join(const Params& p, cudaStream_t stream) {
    // while a block a row is at most one wave of blocks
    return p.total_tokens * p.num_kv_heads * p.group <= 148 * 5 ? launch_join<D, kJoinWarps>(p, stream) : launch_join<D, 1>(p, stream);
}

// ------------------------------------------------------------------ float32
// For checking: a warp per (token, head); four keys a step, eight lanes to a key with D / 8 of its elements each, and a running
// maximum and sum for each of the four, joined at the end of the row.  Bound by that walk.
constexpr int kRowWarps = 4;

template <int D>
__global__ void __launch_bounds__(kRowWarps * 32) group_rows_kernel(const Params p) {
    constexpr int U = D / 8;  // elements of a lane
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, sub = lane >> 3, part = lane & 7;
    bool good = true;
    for (int32_t s = threadIdx.x; s < p.batch; s += blockDim.x) good &= __ldg(p.cu + s) <= __ldg(p.cu + s + 1);
    const bool ordered = __syncthreads_and(good) != 0;
    if (blockIdx.x == 0) {  // what does not fit is reported once
        Seq q;
        for (int32_t s = threadIdx.x; s < p.batch; s += blockDim.x)
            if (!read_seq(p, s, &q)) report(p.status);
        good = ordered;
        for (int32_t g = threadIdx.x; g < p.n_groups; g += blockDim.x) good &= __ldg(p.cu_groups + g) <= __ldg(p.cu_groups + g + 1);
        const bool ascend = __syncthreads_and(good) != 0;
        for (int32_t g = warp; g < p.n_groups; g += kRowWarps) {
            const int32_t first = min(max(__ldg(p.cu_groups + g), 0), p.batch), last = ascend ? min(__ldg(p.cu_groups + g + 1), p.batch) : 0;
            int32_t room = INT32_MAX;
            for (int32_t s = first + lane; s < last; s += 32) {
                if (!read_seq(p, s, &q)) room = -1;
                else if (q.n > 0) room = min(room, q.len - q.n);
            }
            room = __reduce_min_sync(0xffffffffu, room);
            if (lane == 0) {
                const int32_t end = __ldg(p.cu_groups + g + 1);
                const bool fits = group_fits(p, ascend, __ldg(p.cu_groups + g), end, __ldg(p.shared + g), room);
                shared_tokens(p, fits, fits ? __ldg(p.cu + end) - __ldg(p.cu + first) : 0, 0, 0);
            }
        }
    }
    const int64_t row = static_cast<int64_t>(blockIdx.x) * kRowWarps + warp;
    const int64_t token = row / p.num_q_heads;
    const int32_t head = static_cast<int32_t>(row - token * p.num_q_heads);
    if (token >= p.total_tokens || !ordered) return;
    const int32_t s = last_at_or_before(p.cu, p.batch, token, lane);
    Seq seq;
    if (!read_seq(p, s, &seq) || token < seq.tok0 || token - seq.tok0 >= seq.n) return;
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
    for (int64_t j0 = 0; j0 < keys; j0 += 4) {
        const int64_t j = j0 + sub;
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

// A KV head's query heads are taken in as few equal parts as a block has rows for, one after the other: more than 64 are rare.
int32_t part_heads(int32_t step) {
    const int32_t parts = (step + kMostRows - 1) / kMostRows;
    return (step + parts - 1) / parts;
}
// Rows per block: the smallest of 16, 32 and 64 that holds the rows of a KV head of the longest sequence and the largest group, or
// 64, and such blocks side by side.
int32_t choose_cap(const Params& p) {
    const int64_t rows = static_cast<int64_t>(p.n_groups > 0 ? std::max(p.max_q, p.max_group) : p.max_q) * part_heads(p.step);
    return rows <= 16 ? 16 : rows <= 32 ? 32 : kMostRows;
}
constexpr int kMaxCtas = 148;

// Carves the workspace (NULL: only measures it).
size_t carve(Params& p, int32_t head_dim, void* workspace) {
    uint8_t* ws = static_cast<uint8_t*>(workspace);
    size_t at = 0;
    auto take = [&](size_t bytes) {
        uint8_t* r = ws + at;
        at += align_up(bytes, 256);
        return r;
    };
    const size_t rows = static_cast<size_t>(p.total_tokens) * p.num_q_heads * 2, slots = static_cast<size_t>(kMaxCtas) * 2 * p.cap;
    p.entries = reinterpret_cast<Entry*>(take((static_cast<size_t>(p.n_groups) + p.batch) * sizeof(Entry)));
    p.cut = reinterpret_cast<Cut*>(take(sizeof(Cut)));
    p.starts = reinterpret_cast<Start*>(take(kMaxCtas * sizeof(Start)));
    p.whole_ml = reinterpret_cast<float2*>(take(rows * sizeof(float2)));
    p.part_ml = reinterpret_cast<float2*>(take(slots * sizeof(float2)));
    p.whole_o = reinterpret_cast<float*>(take(rows * head_dim * sizeof(float)));
    p.part_o = reinterpret_cast<float*>(take(slots * head_dim * sizeof(float)));
    return at;
}

}  // namespace

int32_t group_most_heads(int32_t head_dim) { return head_dim == 128 ? 112 : 128; }

size_t group_workspace(const rpx_attn_desc_t* d, int64_t tokens, int32_t batch, int32_t n_groups, int32_t max_q, int32_t max_group) {
    if (d->dtype == RPX_F32 || batch > kMostSequences - n_groups) return 0;
    Params p = {};
    p.total_tokens = tokens;
    p.batch = batch;
    p.n_groups = n_groups;
    p.max_q = max_q;
    p.max_group = max_group;
    p.num_q_heads = d->num_q_heads;
    p.step = d->num_q_heads / d->num_kv_heads;
    p.cap = choose_cap(p);
    return carve(p, d->head_dim, nullptr);
}

bool group_too_large(const GroupArgs& a) {
    if ((a.total_tokens * a.num_q_heads + kRowWarps - 1) / kRowWarps > INT32_MAX) return true;
    if (a.num_kv_heads > 65535) return true;  // (a dimension of the join's grid)
    return a.batch > kMostSequences - a.n_groups || a.cache->num_blocks * a.num_kv_heads > INT32_MAX / 2;
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
    p.cap = choose_cap(p);
    p.tile_units = a.head_dim == 128 ? 75 : 38;  // 64 KB or 32 at 6.5 TB/s over 148 SMs
    // (without the SM budget, as the header says: where the line of tiles is cut decides the order of the sums)
    p.ctas = sms < kMaxCtas ? sms : kMaxCtas;
    carve(p, a.head_dim, a.workspace);
    for (int32_t head = 0; head < p.step; head += part_heads(p.step)) {
        p.group = std::min(part_heads(p.step), p.step - head);
        p.group_magic = p.group == 1 ? 0u : static_cast<uint32_t>(((1ull << 32) + p.group - 1) / p.group);
        p.q = static_cast<const __nv_bfloat16*>(a.q) + static_cast<int64_t>(head) * a.head_dim;
        p.out = static_cast<__nv_bfloat16*>(a.out) + static_cast<int64_t>(head) * a.head_dim;
        p.lse = a.lse != nullptr ? a.lse + head : nullptr;
        if (a.n_groups + a.batch <= kPlanThreads) group_plan_small_kernel<<<1, kPlanThreads, 0, a.stream>>>(p);
        else group_plan_kernel<<<1, kPlanThreads, 0, a.stream>>>(p);
        if (cudaGetLastError() != cudaSuccess) return RPX_ERR_CUDA;
        if (rpx_status_t rc = launch_group_tile(p, a.head_dim, *a.cache, a.stream)) return rc;
        if (rpx_status_t rc = a.head_dim == 128 ? launch_join<128>(p, a.stream) : launch_join<64>(p, a.stream)) return rc;
    }
    return RPX_OK;
}

}  // namespace rpx
