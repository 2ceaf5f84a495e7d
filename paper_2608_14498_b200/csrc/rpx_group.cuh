// What the forms of group attention share: the checks of its sequences and groups, and how the work is cut.
//
// All key tiles of all segments lie in a line: first the groups' shared pages (an entry per group), then every sequence's own
// keys (an entry per sequence).  A segment is one KV head of an entry and one block of its rows (row = token * group + head
// within the KV head's group).  The line is cut into equal pieces, one per CTA.  A segment that lies in one piece leaves its
// rows' (maximum in log2 units, sum) and un-normalised outputs in the rows' own place in the workspace (or, where its sequence
// shares nothing, the result in `out`), a segment that is cut one set per piece; the join adds them up in the order of the keys.
// The cut goes by lengths alone, so the same call gives the same bits.
#pragma once

#include <cuda_bf16.h>
#include <math_constants.h>

#include "rpx_internal.h"
#include "rpx_ptx.cuh"

namespace rpx {
namespace group {

constexpr int kPage = 16;
constexpr int kTile = 128;  // keys of a tile
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

// The line is measured in units; going over to another segment counts kSegment of them.
constexpr int kSegment = 10, kMinUnits = 40;

struct __align__(32) Entry {
    int32_t tok0, n, len;   // first query token, query tokens, keys
    int32_t row, page0;     // the table row that names the keys' pages, and the first of them
    int32_t blocks, tiles;  // row blocks, key tiles
    int32_t weight;         // units of a key tile against one block
    __device__ __forceinline__ int32_t block_tokens() const { return (n + blocks - 1) / blocks; }
    __device__ __forceinline__ int64_t segment_units() const { return static_cast<int64_t>(tiles) * weight + kSegment; }
};

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
    // bf16 only
    int32_t cap;           // rows per block at most
    int32_t ctas;          // pieces at most
    Entry* entries;        // workspace [n_groups + batch]
    int64_t* unit0;        // workspace [n_groups + batch + 1]: an entry's first unit; the last is the total
    int32_t* seq_group;    // workspace [batch]: the group whose shared pages a sequence reads, or -1
    float2* whole_ml;      // workspace [2][total_tokens][H_q]: of segments that are not cut: shared, own
    float* whole_o;        // workspace [2][total_tokens][H_q][D]
    float2* part_ml;       // workspace [ctas][2][cap]: of segments that are
    float* part_o;         // workspace [ctas][2][cap][D]
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

// What a group shares: whole pages' tokens, -1 where it does not fit; its first and last sequence, their query tokens, how many
// sequences have any, and the first that does (its table row names the shared pages).  A warp together.
struct Group {
    int32_t first, last, tok0, n, shared, members, row;
};
__device__ __forceinline__ Group read_group(const Params& p, int32_t g, int lane) {
    Group r = {__ldg(p.cu_groups + g), __ldg(p.cu_groups + g + 1), 0, 0, -1, 0, INT32_MAX};
    const int32_t shared = __ldg(p.shared + g);
    if (r.first < 0 || r.last < r.first || r.last > p.batch || shared < 0) return r;
    bool fits = true;
    for (int32_t s = r.first + lane; s < r.last; s += 32) {
        Seq q;
        fits &= read_seq(p, s, &q) && (q.n == 0 || q.len - q.n >= shared);
        if (q.n > 0) {
            ++r.members;
            r.row = min(r.row, s);
        }
    }
    r.members = __reduce_add_sync(0xffffffffu, r.members);
    r.row = __reduce_min_sync(0xffffffffu, r.row);
    if (!__all_sync(0xffffffffu, fits)) return r;
    if (r.first < r.last) {
        r.tok0 = __ldg(p.cu + r.first);
        r.n = __ldg(p.cu + r.last) - r.tok0;
    }
    if (r.n > p.max_group) return r;
    r.shared = shared / kPage * kPage;
    return r;
}

// Pieces: the line of `total` units in runs of piece_units() (the last ones may be short or empty).
__device__ __forceinline__ int64_t piece_units(int64_t total, int32_t ctas) {
    const int64_t even = (total + ctas - 1) / ctas;
    return even > kMinUnits ? even : kMinUnits;
}

// Walks the pieces of segments inside a CTA's part of the line; every role walks it alike.
struct Walk {
    int32_t e, head, block, t0, t1;  // current segment: entry, KV head, row block, key tiles [t0, t1)
    int64_t left;                    // units of the piece behind t1's first
    Entry q, ahead;                  // the entry, and the one behind it
    static __device__ __forceinline__ Entry load(const Params& p, int32_t e) {
        Entry r = {};
        if (e < p.n_groups + p.batch) {
            const int4 a = __ldcg(reinterpret_cast<const int4*>(p.entries + e)), b = __ldcg(reinterpret_cast<const int4*>(p.entries + e) + 1);
            r = Entry{a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
        }
        return r;
    }
    // (a whole warp together)
    __device__ __forceinline__ void start(const Params& p) {
        const int lane = threadIdx.x & 31;
        const int32_t count = p.n_groups + p.batch;
        const int64_t total = __ldcg(p.unit0 + count), size = piece_units(total, p.ctas);
        const int64_t begin = min(total, size * static_cast<int64_t>(blockIdx.x)), end = min(total, begin + size);
        e = head = block = t0 = t1 = 0;
        left = end - begin;
        q = ahead = Entry{};
        if (left == 0) return;
        int32_t lo = 0, hi = count;  // the last entry that starts at or before `begin`, 32 a step
        while (hi - lo > 1) {
            const int32_t step = (hi - lo + 31) / 32;
            const int64_t at = lo + static_cast<int64_t>(lane) * step;
            const uint32_t before = __ballot_sync(0xffffffffu, at < hi && __ldcg(p.unit0 + at) <= begin);
            lo += (before != 0u ? 31 - __clz(static_cast<int>(before)) : 0) * step;
            hi = hi - lo > step ? lo + step : hi;
        }
        e = lo;
        q = load(p, e);
        ahead = load(p, e + 1);
        int64_t off = begin - __ldcg(p.unit0 + e);
        const int64_t seg = q.segment_units(), i = off / seg;
        head = static_cast<int32_t>(i / q.blocks);
        block = static_cast<int32_t>(i - static_cast<int64_t>(head) * q.blocks);
        off -= i * seg;
        t1 = off <= kSegment ? 0 : static_cast<int32_t>((off - kSegment + q.weight - 1) / q.weight);
        left -= kSegment + static_cast<int64_t>(t1) * q.weight - off;
    }
    __device__ __forceinline__ bool next(const Params& p) {
        if (left <= 0) return false;
        if (t1 == q.tiles) {
            t1 = 0;
            if (++block == q.blocks) {
                block = 0;
                if (++head == p.num_kv_heads) {
                    head = 0;
                    do {
                        if (++e >= p.n_groups + p.batch) return false;
                        q = ahead;
                        ahead = load(p, e + 1);
                    } while (q.n == 0);
                }
            }
            left -= kSegment;
            if (left <= 0) return false;  // not even the first tile starts in this piece
        }
        t0 = t1;
        const int64_t tiles = (left + q.weight - 1) / q.weight;
        t1 = tiles < q.tiles - t0 ? t0 + static_cast<int32_t>(tiles) : q.tiles;
        left -= static_cast<int64_t>(t1 - t0) * q.weight;
        return true;
    }
    __device__ __forceinline__ int32_t token0() const { return block * q.block_tokens(); }
    __device__ __forceinline__ int32_t tokens() const { return min(q.block_tokens(), q.n - token0()); }
};

inline Params make_params(const GroupArgs& a) {
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
    return p;
}

}  // namespace group
}  // namespace rpx
