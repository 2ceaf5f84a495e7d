// What the forms of group attention share: the checks of its sequences and groups, and how the work is cut.
//
// All key tiles of all segments lie in a line: first the groups' shared pages (an entry per group), then every sequence's own
// keys (an entry per sequence).  A segment is one KV head of an entry and one block of its rows (row = token * group + head
// within the KV head's group).  The line is cut into equal pieces, one per CTA.  A segment that lies in one piece leaves its rows' (maximum in log2 units, sum) and
// un-normalised outputs in the rows' own place in the workspace (or, where its sequence shares nothing, the result in `out`), a
// segment that is cut one set per piece; the join adds them up in the order of the keys.
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
constexpr int kMostRows = 64;  // of a block
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

// The line is measured in units of some 20 ns; going over to another segment counts kSegment of them (what more it costs is in
// the weight of its tiles).  A piece has kMinUnits at least: as long as the heaviest tile, so every piece between a segment's
// first and last holds one.
constexpr int kSegment = 10, kMinUnits = 192;

struct __align__(16) Entry {
    int32_t tok0, n, len;   // first query token, query tokens, keys
    int32_t row, page0;     // the table row that names the keys' pages, and the first of them
    int32_t blocks, block_tokens;  // row blocks, and the tokens of each but the last
    int32_t weight;         // units of a key tile against one block
    int64_t unit0;          // its first unit, counted from the start of the line
    int32_t group;          // of a sequence: the group whose shared pages it reads as well, or -1
    int32_t tiles;          // key tiles
    __device__ __forceinline__ int64_t segment_units() const { return static_cast<int64_t>(tiles) * weight + kSegment; }
};

__device__ __forceinline__ Entry load_entry(const Entry* at) {
    const int4 a = __ldcg(reinterpret_cast<const int4*>(at)), b = __ldcg(reinterpret_cast<const int4*>(at) + 1);
    const longlong2 c = __ldcg(reinterpret_cast<const longlong2*>(at) + 2);
    return Entry{a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w, c.x, static_cast<int32_t>(c.y), static_cast<int32_t>(c.y >> 32)};
}

struct Start;
struct Cut;

struct Params {
    const void* q;
    int64_t q_stride;
    const int32_t *cu, *lens;
    int32_t batch;
    int64_t total_tokens;
    int32_t max_q, max_group;
    const int32_t *cu_groups, *shared;
    int32_t n_groups;
    int32_t num_q_heads, num_kv_heads, step;  // step: query heads to a KV head
    int32_t group;         // those of them that this pass takes: all, or a part (q, out and lse begin with its first)
    uint32_t group_magic;  // 2^32 / group, rounded up: row / group for rows below 2^16 (group 1: 0)
    const int32_t* block_table;
    int32_t block_table_stride, num_blocks;
    const __nv_bfloat16 *k_cache, *v_cache;
    float scale_log2;
    void* out;
    float* lse;
    int32_t* status;
    // bf16 only
    int32_t tile_units;    // of a tile's bytes
    int32_t ctas;          // pieces of the line at most
    int32_t cap;           // rows per block at most
    Entry* entries;        // workspace [n_groups + batch]
    struct Start* starts;  // workspace [ctas]
    struct Cut* cut;       // workspace
    float2* whole_ml;      // workspace [2][total_tokens][H_q]: of segments that are not cut: shared, own
    float* whole_o;        // workspace [2][total_tokens][H_q][D]
    float2* part_ml;       // workspace [ctas][2][cap]: of segments that are
    float* part_o;         // workspace [ctas][2][cap][D]
};

__device__ __forceinline__ int32_t over_group(const Params& p, int32_t row) {
    return p.group == 1 ? row : static_cast<int32_t>(__umulhi(static_cast<uint32_t>(row), p.group_magic));
}

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

// How the line is cut: the units of a piece (the last ones may be short or empty), and 1 / units.
struct Cut {
    int64_t size;
    double inverse;
};
__device__ __forceinline__ int64_t piece_units(int64_t total, int32_t ctas) {
    const int64_t even = (total + ctas - 1) / ctas;
    return even > kMinUnits ? even : kMinUnits;
}
// The piece that a unit is in.  (A division takes more instructions than the join has otherwise.)
__device__ __forceinline__ int32_t piece_of(int64_t unit, int64_t size, double inverse) {
    int64_t q = static_cast<int64_t>(static_cast<double>(unit) * inverse);
    const int64_t rest = unit - q * size;
    q += rest < 0 ? -1 : rest >= size ? 1 : 0;
    return static_cast<int32_t>(q);
}

__device__ __forceinline__ int64_t quotient(int64_t a, int64_t b) {  // (64-bit division takes ten times as long)
    if ((a >> 31) == 0 && (b >> 31) == 0) return static_cast<uint32_t>(a) / static_cast<uint32_t>(b);
    return a / b;
}

// Where a CTA's piece begins: its entry, KV head, row block and first tile (as Walk keeps them), and the units behind that.
struct __align__(16) Start {
    Entry q;
    int32_t e, head, block, t1;
    int64_t left, unused;
};
// By one thread for one CTA; unit0(e) gives an entry's first unit.
template <class Unit0>
__device__ __forceinline__ Start find_start(const Params& p, int64_t total, int64_t size, int32_t cta, Unit0 unit0) {
    const int64_t begin = min(total, size * static_cast<int64_t>(cta)), end = min(total, begin + size);
    Start r = {};
    r.left = end - begin;
    if (r.left == 0) return r;
    int32_t lo = 0, hi = p.n_groups + p.batch;  // the last entry that starts at or before `begin`
    while (hi - lo > 1) {
        const int32_t mid = lo + (hi - lo) / 2;
        if (unit0(mid) <= begin) lo = mid;
        else hi = mid;
    }
    r.e = lo;
    r.q = p.entries[lo];
    int64_t off = begin - unit0(lo);
    const int64_t seg = r.q.segment_units(), i = quotient(off, seg);
    r.head = static_cast<int32_t>(quotient(i, r.q.blocks));
    r.block = static_cast<int32_t>(i - static_cast<int64_t>(r.head) * r.q.blocks);
    off -= i * seg;
    r.t1 = off <= kSegment ? 0 : static_cast<int32_t>(quotient(off - kSegment + r.q.weight - 1, r.q.weight));
    r.left -= kSegment + static_cast<int64_t>(r.t1) * r.q.weight - off;
    return r;
}

// Walks the pieces of segments inside a CTA's part of the line; every role walks it alike.
struct Walk {
    int32_t e, head, block, t0, t1;  // current segment: entry, KV head, row block, key tiles [t0, t1)
    int32_t left;                    // units of the piece behind t1's first
    Entry q;
    __device__ __forceinline__ void start(const Params& p, int32_t piece) {
        const Start* s = p.starts + piece;
        const int4 a = __ldcg(reinterpret_cast<const int4*>(&s->e));
        left = static_cast<int32_t>(__ldcg(&s->left));  // (2^31 units are 40 s)
        q = load_entry(&s->q);
        e = a.x;
        head = a.y;
        block = a.z;
        t1 = a.w;
        t0 = 0;
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
                        q = load_entry(p.entries + e);
                    } while (q.n == 0);
                }
            }
            left -= kSegment;
            if (left <= 0) return false;  // not even the first tile starts in this piece
        }
        t0 = t1;
        t1 = q.tiles;
        const int64_t all = static_cast<int64_t>(t1 - t0) * q.weight;
        if (all > left) {
            t1 = t0 + (left + q.weight - 1) / q.weight;
            left = 0;
        } else {
            left -= static_cast<int32_t>(all);
        }
        return true;
    }
    __device__ __forceinline__ int32_t token0() const { return block * q.block_tokens; }
    __device__ __forceinline__ int32_t tokens() const { return min(q.block_tokens, q.n - token0()); }
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
    p.step = p.group = a.num_q_heads / a.num_kv_heads;
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
