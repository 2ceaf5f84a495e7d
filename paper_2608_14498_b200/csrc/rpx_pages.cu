// Pages of the paged KV cache: sharing, freeing and compacting them on the device, copying their contents, and storing
// single tokens behind a sequence.  Nothing here is read back by the host, so a captured graph can branch and drop
// sequences whose lengths it does not know.
//
// The bookkeeping is integers: a reference count per page (0 = free) and the block table, of which the held pages of a row
// are entries 0 .. held - 1 and the rest is -1.  Fresh pages are always the free ones with the lowest numbers, in the
// order of the requests, and every decision goes by numbers and not by which block runs first: the same call gives the
// same table.  These kernels are bound by launch and memory latency; the bytes are in the copies, which are a plain
// stream of 16-byte loads and stores.
#include <cuda_bf16.h>

#include "rpx_internal.h"

namespace rpx {

namespace {

constexpr int kPage = 16;

__device__ __forceinline__ void report(int32_t* status, int32_t code) {
    if (status != nullptr) atomicCAS(status, 0, code);
}

// Inclusive sum over a block of `kThreads` threads; `all` receives the total.  `sums` holds kThreads / 32 words.
template <int kThreads, class T>
__device__ __forceinline__ T block_scan(T x, T* sums, T* all) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
    for (int off = 1; off < 32; off <<= 1) {
        const T y = __shfl_up_sync(0xffffffffu, x, off);
        if (lane >= off) x += y;
    }
    __syncthreads();
    if (lane == 31) sums[warp] = x;
    __syncthreads();
    T mine = lane < kThreads / 32 ? sums[lane] : T(0);
#pragma unroll
    for (int off = 1; off < 32; off <<= 1) {
        const T y = __shfl_up_sync(0xffffffffu, mine, off);
        if (lane >= off) mine += y;
    }
    *all = __shfl_sync(0xffffffffu, mine, kThreads / 32 - 1);
    const T before = __shfl_sync(0xffffffffu, mine, warp > 0 ? warp - 1 : 0);
    return x + (warp > 0 ? before : T(0));
}

// ------------------------------------------------------------------ free
// One block per row.  An entry is taken out of the table by an exchange, so a row listed twice gives its pages up once.
__global__ void __launch_bounds__(256) pages_free_kernel(PageArgs a, const int32_t* __restrict__ rows) {
    const int32_t row = __ldg(rows + blockIdx.x);
    if (row < 0 || row >= a.rows) {
        if (threadIdx.x == 0) report(a.device_status, RPX_ERR_DEVICE_DATA);
        return;
    }
    int32_t* entries = a.block_table + static_cast<int64_t>(row) * a.block_table_stride;
    bool bad = false;
    for (int32_t j = threadIdx.x; j < a.table_cols; j += blockDim.x) {
        if (entries[j] < 0) continue;
        const int32_t page = atomicExch(entries + j, -1);
        if (page < 0) continue;
        if (page >= a.num_blocks) {
            bad = true;
        } else if (atomicSub(a.ref_counts + page, 1) <= 0) {  // nobody held it: put the count back
            atomicAdd(a.ref_counts + page, 1);
            bad = true;
        }
    }
    if (threadIdx.x == 0) a.lens[row] = 0;
    if (bad) report(a.device_status, RPX_ERR_DEVICE_DATA);
}

// ------------------------------------------------------------------ fork
struct ForkPlan {  // in the workspace
    int32_t* start;   // [n] number of the request's first fresh page
    int32_t* fresh;   // [n] its fresh pages, -1: the request is refused
    int32_t* owner;   // [rows] twice the request that writes the row (+ 1: a row that only grows)
    int32_t* pages;   // [num_blocks] the lowest free pages
    int32_t* found;   // how many there are (as many as asked for, or all)
};
constexpr int32_t kNobody = 0x7fffffff;
constexpr int kPlanThreads = 1024;
constexpr int kScanInts = 16;  // pages a thread looks at per step

struct ForkRequest {
    int32_t src, dst, len, whole, need, held;  // held: pages the destination has already (grown rows only)
    bool good;
};

__device__ __forceinline__ ForkRequest read_request(const PageArgs& a, const int32_t* src_rows, const int32_t* dst_rows, int32_t extra, int32_t i) {
    ForkRequest r;
    r.src = __ldg(src_rows + i);
    r.dst = __ldg(dst_rows + i);
    r.len = r.whole = r.need = r.held = 0;
    r.good = r.dst >= 0 && r.dst < a.rows && r.src >= -1 && r.src < a.rows;
    if (!r.good) return r;
    if (r.src >= 0) r.len = a.lens[r.src];
    const int64_t need = (static_cast<int64_t>(r.len) + extra + kPage - 1) / kPage;
    const int32_t cached = r.len / kPage + (r.len % kPage != 0 ? 1 : 0);
    r.good = r.len >= 0 && need <= a.table_cols;
    if (!r.good) return r;
    r.need = static_cast<int32_t>(need);
    r.whole = r.len / kPage;
    const int32_t* from = a.block_table + static_cast<int64_t>(r.src < 0 ? 0 : r.src) * a.block_table_stride;
    if (cached > 0 && from[cached - 1] < 0) r.good = false;  // the row does not hold what its length says
    if (r.src == r.dst) {  // held pages are a run from 0: its end by bisection
        int32_t lo = 0, hi = a.table_cols;
        while (lo < hi) {
            const int32_t mid = (lo + hi) >> 1;
            if (from[mid] >= 0) lo = mid + 1;
            else hi = mid;
        }
        r.held = lo;
    } else if (a.table_cols > 0 && (a.block_table[static_cast<int64_t>(r.dst) * a.block_table_stride] >= 0 || a.lens[r.dst] != 0)) {
        r.good = false;  // the destination still holds pages
    }
    return r;
}
__device__ __forceinline__ int32_t fresh_pages(const ForkRequest& r) {
    return max(0, r.need - (r.src == r.dst ? r.held : r.whole));
}

__device__ __forceinline__ void apply_request(const PageArgs& a, const int32_t* src_rows, const int32_t* dst_rows, int32_t extra, const ForkPlan& plan,
                                              int32_t i, int32_t self, int32_t threads, int32_t* copy_src, int32_t* copy_dst);

// One block.  kApply: it also carries the requests out, a warp each (few of them: see launch_pages_fork).
template <bool kApply>
__global__ void __launch_bounds__(kPlanThreads) fork_plan_kernel(PageArgs a, const int32_t* __restrict__ src_rows, const int32_t* __restrict__ dst_rows,
                                                                 int32_t n, int32_t extra, ForkPlan plan, int32_t* copy_src, int32_t* copy_dst) {
    __shared__ int64_t sums[32];
    for (int32_t r = threadIdx.x; r < a.rows; r += kPlanThreads) plan.owner[r] = kNobody;
    __syncthreads();
    for (int32_t i = threadIdx.x; i < n; i += kPlanThreads) {
        const int32_t dst = __ldg(dst_rows + i);
        if (dst >= 0 && dst < a.rows) atomicMin(plan.owner + dst, 2 * i + (__ldg(src_rows + i) == dst ? 1 : 0));
    }
    __syncthreads();
    int64_t carry = 0, all = 0;
    for (int32_t base = 0; base < n; base += kPlanThreads) {
        const int32_t i = base + static_cast<int32_t>(threadIdx.x);
        int32_t fresh = 0;
        if (i < n) {
            ForkRequest r = read_request(a, src_rows, dst_rows, extra, i);
            // a row is written by one request (the first), and no other request reads a row that is forked into
            if (r.good && (plan.owner[r.dst] >> 1) != i) r.good = false;
            if (r.good && r.src >= 0 && r.src != r.dst && plan.owner[r.src] != kNobody && (plan.owner[r.src] & 1) == 0) r.good = false;
            if (!r.good) report(a.device_status, RPX_ERR_DEVICE_DATA);
            fresh = r.good ? fresh_pages(r) : 0;
            plan.fresh[i] = r.good ? fresh : -1;
        }
        const int64_t sum = carry + block_scan<kPlanThreads, int64_t>(fresh, sums, &all);
        if (i < n) plan.start[i] = static_cast<int32_t>(min(sum - fresh, static_cast<int64_t>(kNobody)));  // beyond any pool
        carry += all;
    }
    const int64_t wanted = min(carry, static_cast<int64_t>(a.num_blocks));
    int64_t found = 0;
    for (int64_t base = 0; base < a.num_blocks && found < wanted; base += kPlanThreads * kScanInts) {
        const int64_t first = base + static_cast<int64_t>(threadIdx.x) * kScanInts;
        uint32_t free_mask = 0u;
        if (first + kScanInts <= a.num_blocks && (reinterpret_cast<uintptr_t>(a.ref_counts) & 15u) == 0u) {
            const int4* v = reinterpret_cast<const int4*>(a.ref_counts + first);
#pragma unroll
            for (int k = 0; k < kScanInts / 4; ++k) {
                const int4 c = v[k];
                free_mask |= ((c.x <= 0 ? 1u : 0u) | (c.y <= 0 ? 2u : 0u) | (c.z <= 0 ? 4u : 0u) | (c.w <= 0 ? 8u : 0u)) << (4 * k);
            }
        } else {
            for (int k = 0; k < kScanInts; ++k)
                if (first + k < a.num_blocks && a.ref_counts[first + k] <= 0) free_mask |= 1u << k;
        }
        int64_t at = found + block_scan<kPlanThreads, int64_t>(__popc(free_mask), sums, &all) - __popc(free_mask);
        while (free_mask != 0u && at < wanted) {
            plan.pages[at++] = static_cast<int32_t>(first) + __ffs(static_cast<int>(free_mask)) - 1;
            free_mask &= free_mask - 1;
        }
        found += all;
    }
    if (threadIdx.x == 0) *plan.found = static_cast<int32_t>(min(found, wanted));
    if (kApply) {
        __syncthreads();
        for (int32_t i = threadIdx.x >> 5; i < n; i += kPlanThreads / 32)
            apply_request(a, src_rows, dst_rows, extra, plan, i, threadIdx.x & 31, 32, copy_src, copy_dst);
    }
}

// One request's row of the table, the counts, the pair of pages to copy; by `threads` threads, of which this is number `self`.
__device__ __forceinline__ void apply_request(const PageArgs& a, const int32_t* src_rows, const int32_t* dst_rows, int32_t extra, const ForkPlan& plan,
                                              int32_t i, int32_t self, int32_t threads, int32_t* copy_src, int32_t* copy_dst) {
    const int32_t fresh = plan.fresh[i], start = plan.start[i];
    int32_t from_page = -1, to_page = -1;
    if (fresh > 0 && static_cast<int64_t>(start) + fresh > *plan.found) {
        if (self == 0) report(a.device_status, RPX_ERR_NO_PAGES);
    } else if (fresh >= 0) {
        const int32_t src = __ldg(src_rows + i), dst = __ldg(dst_rows + i);
        const int32_t len = src >= 0 ? a.lens[src] : 0;
        const int32_t whole = len / kPage, need = static_cast<int32_t>((static_cast<int64_t>(len) + extra + kPage - 1) / kPage);
        const bool grows = src == dst;
        const int32_t first = grows ? need - fresh : whole;  // entries from here on are fresh pages
        const int32_t* from = a.block_table + static_cast<int64_t>(src < 0 ? 0 : src) * a.block_table_stride;
        int32_t* to = a.block_table + static_cast<int64_t>(dst) * a.block_table_stride;
        bool bad = false;
        if (!grows)
            for (int32_t j = self; j < whole; j += threads) {
                const int32_t page = from[j];
                to[j] = page;
                if (page >= 0 && page < a.num_blocks) atomicAdd(a.ref_counts + page, 1);
                else bad = true;
            }
        for (int32_t j = self; j < fresh; j += threads) {
            const int32_t page = plan.pages[start + j];
            to[first + j] = page;
            a.ref_counts[page] = 1;
        }
        if (bad) report(a.device_status, RPX_ERR_DEVICE_DATA);
        if (self == 0 && !grows) {
            a.lens[dst] = len;
            if (len % kPage != 0) {
                from_page = from[whole];
                // need > whole here, so the partial page's place is the first fresh page
                to_page = plan.pages[start];
            }
        }
    }
    if (self == 0) {
        copy_src[i] = from_page;
        copy_dst[i] = to_page;
    }
}

__global__ void __launch_bounds__(256) fork_apply_kernel(PageArgs a, const int32_t* __restrict__ src_rows, const int32_t* __restrict__ dst_rows,
                                                         int32_t extra, ForkPlan plan, int32_t* copy_src, int32_t* copy_dst) {
    apply_request(a, src_rows, dst_rows, extra, plan, blockIdx.x, threadIdx.x, blockDim.x, copy_src, copy_dst);
}

// ------------------------------------------------------------------ compact
// With L live pages, the live pages numbered L and above move to the free numbers below L, in order.  Three launches:
// live pages per chunk; every page's place; the table.
constexpr int kChunk = 1024, kChunkThreads = 256, kPerThread = kChunk / kChunkThreads;

__device__ __forceinline__ uint32_t live_mask(const int32_t* ref_counts, int32_t num_blocks, int64_t first) {
    uint32_t m = 0u;
#pragma unroll
    for (int k = 0; k < kPerThread; ++k)
        if (first + k < num_blocks && ref_counts[first + k] > 0) m |= 1u << k;
    return m;
}

__global__ void __launch_bounds__(kChunkThreads) compact_count_kernel(const int32_t* __restrict__ ref_counts, int32_t num_blocks, int32_t* counts) {
    __shared__ int32_t sums[32];
    const int64_t first = static_cast<int64_t>(blockIdx.x) * kChunk + threadIdx.x * kPerThread;
    int32_t all;
    block_scan<kChunkThreads, int32_t>(__popc(live_mask(ref_counts, num_blocks, first)), sums, &all);
    if (threadIdx.x == 0) counts[blockIdx.x] = all;
}

constexpr int32_t kStays = 0x7fffffff;

__global__ void __launch_bounds__(kChunkThreads)
compact_place_kernel(const int32_t* ref_counts, int32_t* ref_counts_out, int32_t num_blocks, const int32_t* __restrict__ counts,
                     int32_t chunks, int32_t* place, int32_t* copy_src, int32_t* copy_dst, int32_t* n_live, int32_t* n_moves) {
    __shared__ int32_t sums[32];
    // live pages in all, before this chunk, and before number L
    int32_t all = 0, before = 0, live = 0, below = 0;
    int32_t mine = 0, mine_before = 0;
    for (int32_t c = threadIdx.x; c < chunks; c += kChunkThreads) {
        mine += counts[c];
        if (c < static_cast<int32_t>(blockIdx.x)) mine_before += counts[c];
    }
    block_scan<kChunkThreads, int32_t>(mine, sums, &live);
    block_scan<kChunkThreads, int32_t>(mine_before, sums, &before);
    const int32_t edge = live / kChunk;  // the chunk that holds number L
    mine = 0;
    for (int32_t c = threadIdx.x; c < chunks && c < edge; c += kChunkThreads) mine += counts[c];
#pragma unroll
    for (int k = 0; k < kPerThread; ++k) {
        const int64_t id = static_cast<int64_t>(edge) * kChunk + threadIdx.x * kPerThread + k;
        if (id < live && id < num_blocks && ref_counts[id] > 0) ++mine;
    }
    block_scan<kChunkThreads, int32_t>(mine, sums, &below);

    const int64_t first = static_cast<int64_t>(blockIdx.x) * kChunk + threadIdx.x * kPerThread;
    const uint32_t mask = live_mask(ref_counts, num_blocks, first);
    int32_t rank = before + block_scan<kChunkThreads, int32_t>(__popc(mask), sums, &all) - __popc(mask);  // live pages before `first`
#pragma unroll
    for (int k = 0; k < kPerThread; ++k) {
        const int64_t id = first + k;
        if (id >= num_blocks) break;
        const bool is_live = ((mask >> k) & 1u) != 0u;
        if (is_live && id >= live) {  // moves: the (rank - below)-th one
            place[id] = rank - below;
            copy_src[rank - below] = static_cast<int32_t>(id);
        } else {
            place[id] = is_live ? kStays : -1;
            if (!is_live && id < live) copy_dst[id - rank] = static_cast<int32_t>(id);  // the (id - rank)-th free number
            ref_counts_out[id] = is_live ? ref_counts[id] : 0;
        }
        rank += is_live ? 1 : 0;
    }
    if (blockIdx.x == 0 && threadIdx.x == 0) {
        *n_live = live;
        *n_moves = live - below;
    }
}

__global__ void __launch_bounds__(256)
compact_table_kernel(PageArgs a, int32_t* table_out, int64_t table_out_stride, int32_t* ref_counts_out, const int32_t* __restrict__ place,
                     const int32_t* __restrict__ n_moves, int32_t max_moves, int32_t* copy_src, int32_t* copy_dst) {
    const int64_t threads = static_cast<int64_t>(gridDim.x) * blockDim.x;
    const int64_t self = static_cast<int64_t>(blockIdx.x) * blockDim.x + threadIdx.x;
    const int32_t moves = *n_moves;
    for (int64_t k = self; k < max_moves; k += threads) {
        if (k < moves) {
            const int32_t from = copy_src[k], to = copy_dst[k];
            const int32_t count = a.ref_counts[from];
            ref_counts_out[to] = count;
            ref_counts_out[from] = 0;
        } else {
            copy_src[k] = copy_dst[k] = -1;
        }
    }
    const int64_t entries = static_cast<int64_t>(a.rows) * a.table_cols;
    bool bad = false;
    for (int64_t e = self; e < entries; e += threads) {
        const int64_t row = e / a.table_cols, col = e - row * a.table_cols;
        int32_t page = a.block_table[row * a.block_table_stride + col];
        if (page >= 0) {
            const int32_t to = page < a.num_blocks ? place[page] : -1;
            if (to < 0) {  // a page that is free, or none of the pool's
                bad = true;
                page = -1;
            } else if (to != kStays) {
                page = copy_dst[to];
            }
        }
        table_out[row * table_out_stride + col] = page;
    }
    if (bad) report(a.device_status, RPX_ERR_DEVICE_DATA);
}

// The same in one block and one launch, for small pools and tables.
constexpr int kSmallThreads = 1024, kSmallPages = 4 * kSmallThreads, kSmallEntries = 8 * kSmallThreads;
__global__ void __launch_bounds__(kSmallThreads)
compact_small_kernel(PageArgs a, int32_t* table_out, int64_t table_out_stride, int32_t* ref_counts_out, int32_t* copy_src, int32_t* copy_dst, int32_t* n_live) {
    __shared__ int32_t sums[32];
    __shared__ int32_t place[kSmallPages];    // of every page: itself, where it goes, or -1 (free)
    __shared__ int32_t hole[kSmallPages / 2]; // free numbers below L
    constexpr int kPer = kSmallPages / kSmallThreads;
    int32_t count[kPer], rank[kPer], live = 0, all;  // rank: live pages before this one
#pragma unroll
    for (int k = 0; k < kPer; ++k) {
        const int32_t id = k * kSmallThreads + static_cast<int32_t>(threadIdx.x);
        count[k] = id < a.num_blocks ? a.ref_counts[id] : 0;
        const int32_t one = count[k] > 0 ? 1 : 0;
        rank[k] = live + block_scan<kSmallThreads, int32_t>(one, sums, &all) - one;
        live += all;
    }
    int32_t mine = 0, below;
#pragma unroll
    for (int k = 0; k < kPer; ++k) {
        const int32_t id = k * kSmallThreads + static_cast<int32_t>(threadIdx.x);
        if (id < live && count[k] > 0) ++mine;
        if (id < live && count[k] <= 0) hole[id - rank[k]] = id;
    }
    block_scan<kSmallThreads, int32_t>(mine, sums, &below);  // (its barriers also order `hole`)
    const int32_t moves = live - below, max_moves = a.num_blocks / 2;
    __syncthreads();
#pragma unroll
    for (int k = 0; k < kPer; ++k) {
        const int32_t id = k * kSmallThreads + static_cast<int32_t>(threadIdx.x);
        if (id >= a.num_blocks) continue;
        int32_t to = count[k] > 0 ? id : -1;
        if (count[k] > 0 && id >= live) {
            const int32_t m = rank[k] - below;
            to = hole[m];
            copy_src[m] = id;
            copy_dst[m] = to;
            ref_counts_out[to] = count[k];
        }
        place[id] = to;
        // a hole that a page moves into was written by that page (every one is); all else keeps its count or is free
        if (id >= live || count[k] > 0) ref_counts_out[id] = to == id ? count[k] : 0;
        if (id >= moves && id < max_moves) copy_src[id] = copy_dst[id] = -1;
    }
    __syncthreads();
    bool bad = false;
    const int32_t entries = a.rows * a.table_cols;
    for (int32_t e = threadIdx.x; e < entries; e += kSmallThreads) {
        const int32_t row = e / a.table_cols, col = e - row * a.table_cols;
        int32_t page = a.block_table[static_cast<int64_t>(row) * a.block_table_stride + col];
        if (page >= 0) {
            page = page < a.num_blocks ? place[page] : -1;
            bad |= page < 0;
        }
        table_out[row * table_out_stride + col] = page;
    }
    if (bad) report(a.device_status, RPX_ERR_DEVICE_DATA);
    if (threadIdx.x == 0) *n_live = live;
}

// ------------------------------------------------------------------ copying pages
// A unit is one page of one tensor of one layer.  Lists may be mostly -1 (a compaction's list is as long as the most it
// could move), so a block first gathers the valid ones among 256 of its units, then streams them.
constexpr int kCopyThreads = 256;

// Chunks c, c + kCopyThreads, .. of a page, kAhead loads in flight; returns the first that is left.
template <int kAhead>
__device__ __forceinline__ int32_t copy_run(const uint4* a, uint4* b, int32_t c, int32_t n) {
    for (; c + (kAhead - 1) * kCopyThreads < n; c += kAhead * kCopyThreads) {
        uint4 x[kAhead];
#pragma unroll
        for (int e = 0; e < kAhead; ++e) x[e] = __ldcs(a + c + e * kCopyThreads);
#pragma unroll
        for (int e = 0; e < kAhead; ++e) __stcs(b + c + e * kCopyThreads, x[e]);
    }
    return c;
}

__global__ void __launch_bounds__(kCopyThreads)
copy_pages_kernel(uint4* k_cache, uint4* v_cache, int64_t layer_stride, int32_t layers, int32_t num_blocks, int32_t page_chunks,
                  const int32_t* __restrict__ src, const int32_t* __restrict__ dst, int64_t n, int32_t* status) {
    __shared__ int32_t sums[32];
    __shared__ int32_t from[kCopyThreads], to[kCopyThreads], part[kCopyThreads];
    const int64_t units = n * layers * 2;
    for (int64_t base = 0; base * gridDim.x < units; base += kCopyThreads) {
        const int64_t u = (base + threadIdx.x) * gridDim.x + blockIdx.x;
        int32_t s = -1, d = -1;
        if (u < units) {
            s = __ldg(src + u / (layers * 2));
            d = __ldg(dst + u / (layers * 2));
            if (s >= num_blocks || d >= num_blocks || (s < 0) != (d < 0)) {
                report(status, RPX_ERR_DEVICE_DATA);
                s = d = -1;
            }
        }
        const bool valid = s >= 0 && d >= 0;
        int32_t count;
        const int32_t at = block_scan<kCopyThreads, int32_t>(valid ? 1 : 0, sums, &count) - 1;
        if (valid) {
            from[at] = s;
            to[at] = d;
            part[at] = static_cast<int32_t>(u % (layers * 2));
        }
        __syncthreads();
        for (int32_t i = 0; i < count; ++i) {
            uint4* pool = ((part[i] & 1) != 0 ? v_cache : k_cache) + (part[i] >> 1) * layer_stride;
            const uint4* a = pool + static_cast<int64_t>(from[i]) * page_chunks;
            uint4* b = pool + static_cast<int64_t>(to[i]) * page_chunks;
            // (8 loads ahead copy 24000-page pools at 91 % of the copy rate, 4 at 90)
            int32_t c = copy_run<8>(a, b, threadIdx.x, page_chunks);
            c = copy_run<4>(a, b, c, page_chunks);
            copy_run<1>(a, b, c, page_chunks);
        }
        __syncthreads();
    }
}

// ------------------------------------------------------------------ single tokens behind a sequence
// One warp per (sequence, i-th appended token): K and V of all its heads, 16 bytes a lane.  Listed tokens of 8 heads of 128:
// 8 x 4096 of them take 52 us in bf16 and 75 us in float32 (78 and 82 % of the copy rate), 256 x 17 10 and 14 us.
__device__ __forceinline__ uint4 load_bf16x8(const __nv_bfloat16* p) { return *reinterpret_cast<const uint4*>(p); }
__device__ __forceinline__ uint4 load_bf16x8(const float* p) {  // rounded to nearest-even, as the prefix pass stores float32
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const __nv_bfloat162 v = __floats2bfloat162_rn(p[2 * i], p[2 * i + 1]);
        w[i] = *reinterpret_cast<const uint32_t*>(&v);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}

template <class T>
__global__ void __launch_bounds__(256) append_kernel(AppendArgs a) {
    const int lane = threadIdx.x & 31;
    const int64_t task = static_cast<int64_t>(blockIdx.x) * 8 + (threadIdx.x >> 5);
    const int64_t s = task / a.max_append;
    const int32_t i = static_cast<int32_t>(task - s * a.max_append);
    if (s >= a.batch) return;
    const int32_t tok0 = __ldg(a.cu + s), n = __ldg(a.cu + s + 1) - tok0;
    const int32_t len = __ldg(a.cached_lens + s);
    if (n == 0) return;
    if (tok0 < 0 || n < 0 || static_cast<int64_t>(tok0) + n > a.n_listed || n > a.max_append || len < 0 ||
        (static_cast<int64_t>(len) + n + kPage - 1) / kPage > a.cache.block_table_stride) {
        if (i == 0 && lane == 0) report(a.device_status, RPX_ERR_DEVICE_DATA);
        return;
    }
    if (i >= n) return;
    const int64_t token = a.token_ids != nullptr ? __ldg(a.token_ids + tok0 + i) : tok0 + i;
    const int64_t pos = static_cast<int64_t>(len) + i;
    const int32_t page = __ldg(a.cache.block_table + s * a.cache.block_table_stride + pos / kPage);
    if (token < 0 || token >= a.total_tokens || page < 0 || page >= a.cache.num_blocks) {
        if (lane == 0) report(a.device_status, RPX_ERR_DEVICE_DATA);
        return;
    }
    const T* k = static_cast<const T*>(a.k) + token * a.k_tok_stride;
    const T* v = static_cast<const T*>(a.v) + token * a.v_tok_stride;
    const int32_t row = a.head_dim / 8;  // 16-byte chunks of one head's row
    const int64_t first = static_cast<int64_t>(page) * a.num_kv_heads * kPage + pos % kPage;
    for (int32_t c = lane; c < a.num_kv_heads * row; c += 32) {
        const int32_t head = c / row;
        const int64_t at = (first + static_cast<int64_t>(head) * kPage) * row + (c - head * row);
        reinterpret_cast<uint4*>(a.cache.k_cache)[at] = load_bf16x8(k + c * 8);
        reinterpret_cast<uint4*>(a.cache.v_cache)[at] = load_bf16x8(v + c * 8);
    }
}

rpx_status_t launched() { return cudaGetLastError() == cudaSuccess ? RPX_OK : RPX_ERR_CUDA; }

}  // namespace

rpx_status_t launch_pages_free(const PageArgs& a, const int32_t* rows, int32_t n) {
    pages_free_kernel<<<static_cast<unsigned>(n), 256, 0, a.stream>>>(a, rows);
    return launched();
}

size_t pages_fork_workspace(int32_t n, int32_t rows, int32_t num_blocks) {
    return (2 * static_cast<size_t>(n) + static_cast<size_t>(rows) + static_cast<size_t>(num_blocks) + 1) * sizeof(int32_t);
}

rpx_status_t launch_pages_fork(const PageArgs& a, const int32_t* src_rows, const int32_t* dst_rows, int32_t n, int32_t extra,
                               int32_t* copy_src, int32_t* copy_dst, void* workspace) {
    ForkPlan plan;
    plan.start = static_cast<int32_t*>(workspace);
    plan.fresh = plan.start + n;
    plan.owner = plan.fresh + n;
    plan.pages = plan.owner + a.rows;
    plan.found = plan.pages + a.num_blocks;
    // a block of its own per request takes a launch more (2.5 us), which up to some thousand table entries is the longer way
    if (static_cast<int64_t>(n) * a.table_cols <= 8192) {
        fork_plan_kernel<true><<<1, kPlanThreads, 0, a.stream>>>(a, src_rows, dst_rows, n, extra, plan, copy_src, copy_dst);
        return launched();
    }
    fork_plan_kernel<false><<<1, kPlanThreads, 0, a.stream>>>(a, src_rows, dst_rows, n, extra, plan, copy_src, copy_dst);
    if (rpx_status_t rc = launched()) return rc;
    fork_apply_kernel<<<static_cast<unsigned>(n), 256, 0, a.stream>>>(a, src_rows, dst_rows, extra, plan, copy_src, copy_dst);
    return launched();
}

size_t pages_compact_workspace(int32_t num_blocks) {
    return (static_cast<size_t>(num_blocks) + (static_cast<size_t>(num_blocks) + kChunk - 1) / kChunk + 1) * sizeof(int32_t);
}

rpx_status_t launch_pages_compact(const PageArgs& a, int32_t* table_out, int64_t table_out_stride, int32_t* ref_counts_out,
                                  int32_t* copy_src, int32_t* copy_dst, int32_t* n_live, void* workspace) {
    if (a.num_blocks <= kSmallPages && static_cast<int64_t>(a.rows) * a.table_cols <= kSmallEntries) {
        compact_small_kernel<<<1, kSmallThreads, 0, a.stream>>>(a, table_out, table_out_stride, ref_counts_out, copy_src, copy_dst, n_live);
        return launched();
    }
    const int32_t chunks = (a.num_blocks + kChunk - 1) / kChunk;
    int32_t* place = static_cast<int32_t*>(workspace);
    int32_t* counts = place + a.num_blocks;
    int32_t* n_moves = counts + chunks;
    const int sms = sm_count();
    if (sms <= 0) return RPX_ERR_CUDA;
    compact_count_kernel<<<static_cast<unsigned>(chunks), kChunkThreads, 0, a.stream>>>(a.ref_counts, a.num_blocks, counts);
    if (rpx_status_t rc = launched()) return rc;
    compact_place_kernel<<<static_cast<unsigned>(chunks), kChunkThreads, 0, a.stream>>>(a.ref_counts, ref_counts_out, a.num_blocks, counts, chunks, place,
                                                                                       copy_src, copy_dst, n_live, n_moves);
    if (rpx_status_t rc = launched()) return rc;
    const int32_t max_moves = a.num_blocks / 2;
    const int64_t most = static_cast<int64_t>(a.rows) * a.table_cols > max_moves ? static_cast<int64_t>(a.rows) * a.table_cols : max_moves;
    int64_t blocks = (most + 255) / 256;
    if (blocks < 1) blocks = 1;
    if (blocks > sms * 8) blocks = sms * 8;
    compact_table_kernel<<<static_cast<unsigned>(blocks), 256, 0, a.stream>>>(a, table_out, table_out_stride, ref_counts_out, place, n_moves, max_moves,
                                                                             copy_src, copy_dst);
    return launched();
}

rpx_status_t launch_copy_pages(const CopyPagesArgs& a) {
    const int sms = sm_count();
    if (sms <= 0) return RPX_ERR_CUDA;
    const int64_t units = a.n * a.layers * 2;
    int64_t blocks = static_cast<int64_t>(sms) * 8;
    if (blocks > units) blocks = units;
    copy_pages_kernel<<<static_cast<unsigned>(blocks), kCopyThreads, 0, a.stream>>>(
        static_cast<uint4*>(a.k_cache), static_cast<uint4*>(a.v_cache), a.layer_stride / 8, a.layers, a.num_blocks,
        a.num_kv_heads * kPage * a.head_dim / 8, a.src, a.dst, a.n, a.device_status);
    return launched();
}

rpx_status_t launch_append(const AppendArgs& a) {
    const int64_t blocks = (static_cast<int64_t>(a.batch) * a.max_append + 7) / 8;
    if (blocks > INT32_MAX) return RPX_ERR_SHAPE;
    if (a.dtype == RPX_F32) append_kernel<float><<<static_cast<unsigned>(blocks), 256, 0, a.stream>>>(a);
    else append_kernel<__nv_bfloat16><<<static_cast<unsigned>(blocks), 256, 0, a.stream>>>(a);
    return launched();
}

}  // namespace rpx
