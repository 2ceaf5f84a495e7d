// What the two forms of tree attention share: how the work is cut.
//
// All key tiles of all (sequence, head, row block) segments lie in a line; the line is cut into equal
// pieces, one per CTA of a resident wave.  A segment that lies in one piece is written by its CTA; of a segment that is
// cut, every piece leaves its rows' (maximum in log2 units, sum) and un-normalised outputs in the workspace, and the
// join adds them up in the order of the keys.  The cut goes by lengths alone, so the same call gives the same bits.
#pragma once

#include <cuda_bf16.h>
#include <math_constants.h>

#include "rpx_internal.h"
#include "rpx_ptx.cuh"

namespace rpx {
namespace tree {

constexpr int kPage = 16;
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;
constexpr float kRaise = 8.0f;  // a row's running maximum is raised when a score passes it by this much (log2 units)

struct Params {
    const __nv_bfloat16* q;
    int64_t q_stride;
    const int32_t *cu, *parents, *lens;
    const int32_t* block_table;
    int32_t block_table_stride, num_blocks;
    int32_t batch, num_q_heads, num_kv_heads, group, max_tree;
    int64_t total_tokens;
    int32_t ctas;          // pieces the line is cut into at most (the grid)
    int32_t whole_blocks;  // > 0: short sequences, a CTA per segment (this many blocks per head) and nothing to join
    int32_t tile_nodes;    // tensor-core form: nodes per query tile of 128 rows (128 / group)
    const __nv_bfloat16 *k_cache, *v_cache;
    const uint32_t* sets;  // tensor-core form: ancestor sets [tokens][set_words]
    int32_t set_words;
    float scale_log2;
    __nv_bfloat16* out;    // [tokens][H_q][D]
    float* lse;            // nullable
    int64_t* seq_unit0;    // workspace [batch + 1]: number of the sequence's first unit; the last entry is the total
    float2* part_ml;       // workspace [ctas][2][rows per block]; a negative sum marks a node that is not in use
    float* part_o;         // workspace [ctas][2][rows per block][D], each form in an order of its own (part_at)
    int32_t* status;
};

// How a form cuts: keys per tile, rows of a block (in the workspace), blocks of a sequence, a row's place in its block, and
// the weight of a block's key tiles: the line is measured in units of these, with kSegment units in front of every segment
// for going over to it (its Q, the outputs of the one before), and a tile belongs to the piece that holds its first unit.
// All blocks but a sequence's last have the same weight.
template <int kRows_>
struct RowCut {  // blocks of kRows rows, row = node * group + head within the KV head's group
    static constexpr int kTile = 64, kRows = kRows_, kMinUnits = 3, kSegment = 1, kWholeTiles = kRows_ == 64 ? 3 : 6;
    static __device__ __forceinline__ int32_t weight(const Params&, int32_t, int32_t) { return 1; }
    static __host__ __device__ __forceinline__ int32_t blocks(const Params& p, int32_t n) { return (n * p.group + kRows - 1) / kRows; }
    static __device__ __forceinline__ void place(const Params& p, int32_t node, int32_t h, int32_t* block, int32_t* row) {
        const int32_t r = node * p.group + h;
        *block = r / kRows;
        *row = r % kRows;
    }
    template <int D>
    static __device__ __forceinline__ int64_t part_at(int64_t row, int32_t col) { return row * D + col; }
};
template <int kTiles>
struct NodeCut {  // blocks of kTiles query tiles of tile_nodes nodes each
    static constexpr int kTile = 128, kRows = 128 * kTiles, kWholeTiles = 8;
    // by a fit over the CTAs, a key tile against two query tiles takes 1.67 us, against one 1.0 - 1.35, and going over to
    // another segment 4.5 - 6.5.  The times hardly turn on it: over five batches (8 x 8, 16 x 24, 32 ragged x 16, 12 x 60 and
    // 8 x 192 nodes) weights of (6, 5, 17), (8, 5, 17), (7, 5, 11), (7, 5, 25), (7, 5, 34) and (6, 5, 30) are up to 1.5 % faster
    // and up to 7 % slower with head_dim 64, where a tile has half the bytes, and within the noise or slower with 128.
    static constexpr int kPairWeight = 7, kOneWeight = 5, kSegment = 17;
    static constexpr int kMinUnits = kSegment + 2 * (kTiles == 1 ? kOneWeight : kPairWeight);
    static __device__ __forceinline__ int32_t weight(const Params& p, int32_t n, int32_t block) {
        if (kTiles == 1) return kOneWeight;
        return n - block * kTiles * p.tile_nodes > p.tile_nodes ? kPairWeight : kOneWeight;
    }
    static __host__ __device__ __forceinline__ int32_t blocks(const Params& p, int32_t n) {
        return (n + kTiles * p.tile_nodes - 1) / (kTiles * p.tile_nodes);
    }
    static __device__ __forceinline__ void place(const Params& p, int32_t node, int32_t h, int32_t* block, int32_t* row) {
        const int32_t tile = node / p.tile_nodes;
        *block = tile / kTiles;
        *row = (tile % kTiles) * 128 + (node - tile * p.tile_nodes) * p.group + h;
    }
    // [32 rows][8 columns of each], so that what the 32 lanes of a warp hold of their rows goes out as whole lines: with a row's
    // columns in one run every store touched 32 lines, and the next load waited 4000 clocks behind them
    template <int D>
    static __device__ __forceinline__ int64_t part_at(int64_t row, int32_t col) {
        return ((row >> 5) * (D / 8) + (col >> 3)) * 256 + (row & 31) * 8 + (col & 7);
    }
};

struct Seq {
    int32_t tok0, n, len;         // first token, nodes, cached tokens
    int32_t cached_tiles, tiles;  // key tiles of one segment: cached ones, then the tree's own
    int32_t blocks;               // row blocks
    int32_t weight, last_weight;  // of the key tiles of all blocks but the last, and of the last
    __device__ __forceinline__ int32_t block_weight(int32_t block) const { return block + 1 < blocks ? weight : last_weight; }
};

// What is read of a sequence.
struct SeqRaw {
    int32_t begin, end, len;
};
__device__ __forceinline__ SeqRaw load_seq(const Params& p, int32_t s) { return SeqRaw{__ldg(p.cu + s), __ldg(p.cu + s + 1), __ldg(p.lens + s)}; }

// Units of a whole segment, of a head's segments, of a sequence.
template <class Cut>
__device__ __forceinline__ int64_t segment_units(const Seq& q, int32_t block) {
    return static_cast<int64_t>(q.tiles) * q.block_weight(block) + Cut::kSegment;
}
template <class Cut>
__device__ __forceinline__ int64_t head_units(const Seq& q) {
    return (q.blocks - 1) * segment_units<Cut>(q, 0) + segment_units<Cut>(q, q.blocks - 1);
}
template <class Cut>
__device__ __forceinline__ int64_t seq_units(const Params& p, const Seq& q) { return q.n > 0 ? head_units<Cut>(q) * p.num_kv_heads : 0; }
// A tile's first unit, counted from the start of its segment.
template <class Cut>
__device__ __forceinline__ int64_t tile_unit(const Seq& q, int32_t block, int32_t tile) {
    return Cut::kSegment + static_cast<int64_t>(tile) * q.block_weight(block);
}

// Offsets that leave the packed tensors or the block table, and a tree larger than the caller's bound, make a sequence
// count as empty (its rows are left as they were) and are reported.
template <class Cut>
__device__ __forceinline__ Seq make_seq(const Params& p, const SeqRaw& raw, uint32_t* data_error) {
    Seq q;
    q.tok0 = raw.begin;
    q.n = raw.end - raw.begin;
    q.len = raw.len;
    const bool bad = q.tok0 < 0 || q.n < 0 || static_cast<int64_t>(q.tok0) + q.n > p.total_tokens || q.n > p.max_tree ||
                     (q.n > 0 && (q.len < 0 || (static_cast<int64_t>(q.len) + kPage - 1) / kPage > p.block_table_stride));
    if (bad) {
        if (data_error != nullptr) *data_error = 1;
        q.n = 0;
    }
    if (q.n == 0) q.len = 0;
    q.cached_tiles = q.len / Cut::kTile + (q.len % Cut::kTile != 0 ? 1 : 0);
    q.tiles = q.n > 0 ? q.cached_tiles + (q.n + Cut::kTile - 1) / Cut::kTile : 0;
    q.blocks = Cut::blocks(p, q.n);
    q.weight = Cut::weight(p, q.n, 0);
    q.last_weight = q.n > 0 ? Cut::weight(p, q.n, q.blocks - 1) : q.weight;
    if (seq_units<Cut>(p, q) > INT32_MAX) {  // beyond any memory; the walk counts a sequence's units in 32 bits
        if (data_error != nullptr) *data_error = 1;
        q.n = q.len = q.cached_tiles = q.tiles = q.blocks = 0;
    }
    return q;
}
template <class Cut>
__device__ __forceinline__ Seq read_seq(const Params& p, int32_t s, uint32_t* data_error) {
    return make_seq<Cut>(p, load_seq(p, s), data_error);
}

// The line of `total` units is cut into pieces of piece_units() units (the last ones may be short or empty; none is
// otherwise shorter than a tile's weight, so every piece between a segment's first and last holds a tile).
template <class Cut>
__device__ __forceinline__ int64_t piece_units(int64_t total, int32_t ctas) {
    const int64_t even = (total >> 31) == 0 ? (static_cast<uint32_t>(total) + ctas - 1u) / static_cast<uint32_t>(ctas) : (total + ctas - 1) / ctas;
    return even > Cut::kMinUnits ? even : Cut::kMinUnits;
}
__device__ __forceinline__ int32_t piece_of(int64_t unit, int64_t size) {
    if ((unit >> 31) == 0 && (size >> 31) == 0) return static_cast<int32_t>(static_cast<uint32_t>(unit) / static_cast<uint32_t>(size));
    return static_cast<int32_t>(unit / size);
}

__device__ __forceinline__ int64_t warp_scan(int64_t x, int lane) {  // inclusive
#pragma unroll
    for (int off = 1; off < 32; off <<= 1) {
        const int64_t y = __shfl_up_sync(0xffffffffu, x, off);
        if (lane >= off) x += y;
    }
    return x;
}
// A piece: its first unit (sequence, and unit within that sequence's work) and how many units it has.
struct Piece {
    int32_t seq, off, units;
};

// Finds this CTA's piece; every warp of it works it out by itself (32 sequences a step), so nothing is waited for.  CTA 0's
// first warp also leaves every sequence's first unit in the workspace, and reports bad offsets.
template <class Cut>
__device__ __forceinline__ Piece find_piece(const Params& p, uint32_t* data_error) {
    const int lane = threadIdx.x & 31;
    const bool scribe = blockIdx.x == 0 && threadIdx.x < 32;
    Piece piece = {p.batch, 0, 0};
    if (p.whole_blocks > 0) {
        const int32_t per_seq = p.num_kv_heads * p.whole_blocks, s = blockIdx.x / per_seq, i = blockIdx.x - s * per_seq;
        const int32_t head = i / p.whole_blocks, block = i - head * p.whole_blocks;
        const Seq q = read_seq<Cut>(p, s, i == 0 ? data_error : nullptr);
        if (q.n > 0 && block < q.blocks) {
            piece.seq = s;
            piece.off = static_cast<int32_t>(head * head_units<Cut>(q) + block * segment_units<Cut>(q, 0));
            piece.units = static_cast<int32_t>(segment_units<Cut>(q, block));
        }
        return piece;
    }
    int64_t total = 0, first_work = 0, first_sum = 0;
    for (int32_t base = 0; base < p.batch; base += 32) {
        const int64_t w = base + lane < p.batch ? seq_units<Cut>(p, read_seq<Cut>(p, base + lane, scribe ? data_error : nullptr)) : 0;
        const int64_t sum = total + warp_scan(w, lane);
        if (base == 0) {
            first_work = w;
            first_sum = sum;
        }
        total = __shfl_sync(0xffffffffu, sum, 31);
    }
    const int64_t size = piece_units<Cut>(total, p.ctas);
    const int64_t begin = min(total, size * static_cast<int64_t>(blockIdx.x)), end = min(total, begin + size);
    int64_t carry = 0;
    for (int32_t base = 0; base < p.batch; base += 32) {
        int64_t w = first_work, sum = first_sum;
        if (base > 0) {
            w = base + lane < p.batch ? seq_units<Cut>(p, read_seq<Cut>(p, base + lane, nullptr)) : 0;
            sum = carry + warp_scan(w, lane);
        }
        const int64_t before = sum - w;
        const uint32_t found = __ballot_sync(0xffffffffu, begin < end && begin >= before && begin < sum);
        if (found != 0u) {
            const int src = __ffs(static_cast<int>(found)) - 1;
            piece.seq = base + src;
            piece.off = static_cast<int32_t>(begin - __shfl_sync(0xffffffffu, before, src));
            piece.units = static_cast<int32_t>(end - begin);
            if (!scribe) break;
        }
        if (scribe && base + lane < p.batch) p.seq_unit0[base + lane] = before;
        carry = __shfl_sync(0xffffffffu, sum, 31);
    }
    if (scribe && lane == 0) p.seq_unit0[p.batch] = total;
    return piece;
}

// Walks the pieces of segments inside this CTA's part of the line; every warp walks it alike.
template <class Cut>
struct Walk {
    int32_t s, head, block, t0, t1;  // current segment: sequence, KV head, row block, key tiles [t0, t1)
    int32_t left;                    // units of the piece behind t1's first
    Seq q;
    int32_t next_begin, next_end, next_len;  // the sequence behind, read a sequence ahead
    __device__ __forceinline__ void look_ahead(const Params& p) {
        next_end = s + 1 < p.batch ? __ldg(p.cu + s + 2) : 0;
        next_len = s + 1 < p.batch ? __ldg(p.lens + s + 1) : 0;
    }
    __device__ __forceinline__ Walk(const Params& p, const Piece& piece) : s(piece.seq), head(0), block(0), t0(0), t1(0), left(piece.units), q(), next_begin(0), next_end(0), next_len(0) {
        if (left == 0) return;
        const SeqRaw raw = load_seq(p, s);
        look_ahead(p);
        q = make_seq<Cut>(p, raw, nullptr);
        next_begin = raw.end;
        const int32_t per_head = static_cast<int32_t>(head_units<Cut>(q)), per_block = static_cast<int32_t>(segment_units<Cut>(q, 0));
        head = piece.off / per_head;
        int32_t off = piece.off - head * per_head;
        block = min(off / per_block, q.blocks - 1);
        off -= block * per_block;
        const int32_t w = q.block_weight(block);
        t1 = max(0, (off - Cut::kSegment + w - 1) / w);
        left -= Cut::kSegment + t1 * w - off;
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
                        if (++s >= p.batch) return false;
                        const SeqRaw raw = {next_begin, next_end, next_len};
                        look_ahead(p);
                        q = make_seq<Cut>(p, raw, nullptr);
                        next_begin = raw.end;
                    } while (q.n == 0);
                }
            }
            left -= Cut::kSegment;
            if (left <= 0) return false;  // not even the first tile starts in this piece
        }
        const int32_t w = q.block_weight(block);
        t0 = t1;
        t1 = min(q.tiles, t0 + (left + w - 1) / w);
        left -= (t1 - t0) * w;
        return true;
    }
};

// Adds up the pieces of every row whose segment was cut, in an order that the lengths fix.  A warp takes kJoinRows rows (node,
// query head) of a sequence side by side, or, where a handful of rows has dozens of pieces, the eight warps of a block one row,
// each every eighth piece.  Launched on top of the attention kernel.
constexpr int kJoinWarps = 8;

template <int D, class Cut, int kSplit, int kJoinRows>
__global__ void __launch_bounds__(kJoinWarps * 32, kSplit > 1 ? 2 : 4) tree_join_kernel(const Params p, int32_t chunks) {
    constexpr int kCols = D / 32;
    __shared__ float part_acc[kSplit > 1 ? kJoinWarps : 1][kJoinRows][D];
    __shared__ float2 part_row[kSplit > 1 ? kJoinWarps : 1][kJoinRows];  // (maximum, sum); a negative sum: not in use
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, sub = warp % kSplit;
    const int32_t s = blockIdx.x / chunks;
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int64_t total = p.seq_unit0[p.batch], seq0 = p.seq_unit0[s];  // (in flight together with the lengths)
    const Seq q = read_seq<Cut>(p, s, nullptr);
    const int32_t row_begin = ((blockIdx.x - s * chunks) * (kJoinWarps / kSplit) + warp / kSplit) * kJoinRows, rows = q.n * p.num_q_heads;
    if (row_begin >= rows && kSplit == 1) return;
    const int64_t size = piece_units<Cut>(total, p.ctas);
    {
        int32_t c0[kJoinRows], n[kJoinRows], row[kJoinRows], most = 0;  // first piece, pieces (0: nothing to do), place in a slot
#pragma unroll
        for (int k = 0; k < kJoinRows; ++k) {
            c0[k] = n[k] = row[k] = 0;
            if (row_begin + k < rows) {
                const int32_t node = (row_begin + k) / p.num_q_heads, head = row_begin + k - node * p.num_q_heads, kv_head = head / p.group;
                int32_t block;
                Cut::place(p, node, head - kv_head * p.group, &block, &row[k]);
                const int64_t unit0 = seq0 + kv_head * head_units<Cut>(q) + block * segment_units<Cut>(q, 0);
                c0[k] = piece_of(unit0 + tile_unit<Cut>(q, block, 0), size);
                n[k] = piece_of(unit0 + tile_unit<Cut>(q, block, q.tiles - 1), size) - c0[k] + 1;
                if (n[k] == 1) n[k] = 0;  // written whole
                most = max(most, n[k]);
            }
        }
        if (kSplit == 1 && most == 0) return;
        float top[kJoinRows], sum[kJoinRows], acc[kJoinRows][kCols];
        bool unused[kJoinRows];
#pragma unroll
        for (int k = 0; k < kJoinRows; ++k) {
            top[k] = -CUDART_INF_F;
            sum[k] = 0.f;
            unused[k] = false;
#pragma unroll
            for (int e = 0; e < kCols; ++e) acc[k][e] = 0.f;
        }
#pragma unroll (kSplit > 1 ? 8 : 2)
        for (int32_t j = sub; j < most; j += kSplit) {
            float2 ml[kJoinRows];
            float4 v[kJoinRows];
#pragma unroll
            for (int k = 0; k < kJoinRows; ++k) {
                ml[k] = make_float2(-CUDART_INF_F, 0.f);
                v[k] = make_float4(0.f, 0.f, 0.f, 0.f);
                if (j < n[k]) {
                    // a piece keeps the segment it starts in the middle of in its first slot, the one it breaks off in its second
                    const int64_t at = (static_cast<int64_t>(c0[k] + j) * 2 + (j == 0 ? 1 : 0)) * Cut::kRows + row[k];
                    ml[k] = p.part_ml[at];
                    if (kCols == 4) {
                        v[k] = *reinterpret_cast<const float4*>(p.part_o + Cut::template part_at<D>(at, lane * kCols));
                    } else {
                        const float2 x = *reinterpret_cast<const float2*>(p.part_o + Cut::template part_at<D>(at, lane * kCols));
                        v[k].x = x.x;
                        v[k].y = x.y;
                    }
                }
            }
#pragma unroll
            for (int k = 0; k < kJoinRows; ++k) {
                unused[k] |= ml[k].y < 0.f;
                if (ml[k].x == -CUDART_INF_F && ml[k].y == ml[k].y) continue;  // no key seen (a NaN sum: nothing but NaN, and goes on)
                const float to = fmaxf(top[k], ml[k].x);
                const float keep = fast_exp2(top[k] - to), f = fast_exp2(ml[k].x - to);
                top[k] = to;
                sum[k] = fmaf(sum[k], keep, f * ml[k].y);
                const float x[4] = {v[k].x, v[k].y, v[k].z, v[k].w};
#pragma unroll
                for (int e = 0; e < kCols; ++e) acc[k][e] = fmaf(acc[k][e], keep, f * x[e]);
            }
        }
        if (kSplit > 1) {
#pragma unroll
            for (int k = 0; k < kJoinRows; ++k) {
#pragma unroll
                for (int e = 0; e < kCols; ++e) part_acc[warp][k][lane * kCols + e] = acc[k][e];
                if (lane == 0) part_row[warp][k] = make_float2(top[k], unused[k] ? -1.f : sum[k]);
            }
            __syncthreads();
            // the first warp finishes the row
#pragma unroll
            for (int k = 0; k < kJoinRows; ++k) {
                if (warp != 0) continue;
                top[k] = -CUDART_INF_F;
                sum[k] = 0.f;
#pragma unroll
                for (int e = 0; e < kCols; ++e) acc[k][e] = 0.f;
#pragma unroll
                for (int w = 0; w < kJoinWarps; ++w) top[k] = fmaxf(top[k], part_row[w][k].x);
#pragma unroll
                for (int w = 0; w < kJoinWarps; ++w) {
                    const float2 ml = part_row[w][k];
                    unused[k] |= ml.y < 0.f;
                    const float f = ml.x == -CUDART_INF_F ? 0.f : fast_exp2(ml.x - top[k]);
                    sum[k] = fmaf(f, ml.y, sum[k]);
#pragma unroll
                    for (int e = 0; e < kCols; ++e) acc[k][e] = fmaf(f, part_acc[w][k][lane * kCols + e], acc[k][e]);
                }
            }
            __syncthreads();
        }
#pragma unroll
        for (int k = 0; k < kJoinRows; ++k) {
            if (n[k] == 0 || (kSplit > 1 && warp != 0)) continue;
            const float inv = unused[k] ? 0.f : 1.f / sum[k];
            const int64_t out_row = static_cast<int64_t>(q.tok0) * p.num_q_heads + row_begin + k;
            uint32_t w[kCols / 2];
#pragma unroll
            for (int e = 0; e < kCols / 2; ++e) w[e] = unused[k] ? 0u : pack_bf16x2(acc[k][2 * e] * inv, acc[k][2 * e + 1] * inv);
            uint32_t* dst = reinterpret_cast<uint32_t*>(p.out + out_row * D + lane * kCols);
            if (kCols == 4) *reinterpret_cast<uint2*>(dst) = make_uint2(w[0], w[kCols / 2 - 1]);
            else *dst = w[0];
            if (lane == 0 && p.lse != nullptr) p.lse[out_row] = unused[k] ? -CUDART_INF_F : (top[k] + log2f(sum[k])) * kLn2;
        }
    }
}

// The same for the tensor-core form with a few pieces to a segment: its rows lie 32 side by side (part_at), so a lane takes a
// row and a warp 32 rows of one segment and kCols of their columns: what it loads are whole kilobytes, and the segment's
// pieces are worked out once.  (8 x 192 nodes over 8192 tokens: 10 us behind the attention kernel; with a warp a row every load
// touched 16 lines, 20 us.  Half the columns a warp, twice the warps: no difference.)
template <int D, int kTiles>
__global__ void __launch_bounds__(kJoinWarps * 32, 2) tree_join_tiles_kernel(const Params p, int32_t blocks) {
    using Cut = NodeCut<kTiles>;
    constexpr int kCols = 32, kParts = D / kCols, kPerSegment = Cut::kRows / 32 * kParts / kJoinWarps;  // CTAs to a segment
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int32_t segment = blockIdx.x / kPerSegment, unit = (blockIdx.x - segment * kPerSegment) * kJoinWarps + warp;
    const int32_t row = unit / kParts * 32 + lane, col0 = unit % kParts * kCols;
    const int32_t block = segment % blocks, kv_head = segment / blocks % p.num_kv_heads, s = segment / blocks / p.num_kv_heads;
    const int32_t tile = row >> 7, in_tile = (row & 127) / p.group, node = (block * kTiles + tile) * p.tile_nodes + in_tile;
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int64_t total = p.seq_unit0[p.batch], seq0 = p.seq_unit0[s];  // (in flight together with the lengths)
    const Seq q = read_seq<Cut>(p, s, nullptr);
    const bool valid = in_tile < p.tile_nodes && node < q.n;
    if (block >= q.blocks || __ballot_sync(0xffffffffu, valid) == 0u) return;
    const int64_t size = piece_units<Cut>(total, p.ctas);
    const int64_t unit0 = seq0 + kv_head * head_units<Cut>(q) + block * segment_units<Cut>(q, 0);
    const int32_t c0 = piece_of(unit0 + tile_unit<Cut>(q, block, 0), size);
    const int32_t n = piece_of(unit0 + tile_unit<Cut>(q, block, q.tiles - 1), size) - c0 + 1;
    if (n == 1 || !valid) return;  // written whole; a row that is nobody's
    float top = -CUDART_INF_F, sum = 0.f, acc[kCols];
    bool unused = false;
#pragma unroll
    for (int e = 0; e < kCols; ++e) acc[e] = 0.f;
#pragma unroll 2
    for (int32_t j = 0; j < n; ++j) {
        // a piece keeps the segment it starts in the middle of in its first slot, the one it breaks off in its second
        const int64_t at = (static_cast<int64_t>(c0 + j) * 2 + (j == 0 ? 1 : 0)) * Cut::kRows + row;
        const float2 ml = p.part_ml[at];
        float v[kCols / 8][8];
#pragma unroll
        for (int c = 0; c < kCols / 8; ++c) ld_global_v8(p.part_o + Cut::template part_at<D>(at, col0 + 8 * c), v[c]);
        unused |= ml.y < 0.f;
        if (ml.x == -CUDART_INF_F && ml.y == ml.y) continue;  // no key seen (a NaN sum: nothing but NaN, and goes on)
        const float to = fmaxf(top, ml.x);
        const float keep = fast_exp2(top - to), f = fast_exp2(ml.x - to);
        top = to;
        sum = fmaf(sum, keep, f * ml.y);
#pragma unroll
        for (int e = 0; e < kCols; ++e) acc[e] = fmaf(acc[e], keep, f * v[e / 8][e % 8]);
    }
    const float inv = unused ? 0.f : 1.f / sum;
    const int64_t out_row = (static_cast<int64_t>(q.tok0) + node) * p.num_q_heads + kv_head * p.group + ((row & 127) - in_tile * p.group);
    uint32_t w[kCols / 2];
#pragma unroll
    for (int e = 0; e < kCols / 2; ++e) w[e] = unused ? 0u : pack_bf16x2(acc[2 * e] * inv, acc[2 * e + 1] * inv);
    uint4* dst = reinterpret_cast<uint4*>(p.out + out_row * D + col0);
#pragma unroll
    for (int i = 0; i < kCols / 8; ++i) dst[i] = make_uint4(w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]);
    if (col0 == 0 && p.lse != nullptr) p.lse[out_row] = unused ? -CUDART_INF_F : (top + log2f(sum)) * kLn2;
}

template <int D, class Cut, int kSplit, int kJoinRows>
rpx_status_t launch_join_split(const Params& p, cudaStream_t stream) {
    constexpr int per_block = kJoinWarps / kSplit * kJoinRows;
    const int64_t chunks = (static_cast<int64_t>(p.max_tree) * p.num_q_heads + per_block - 1) / per_block;
    if (chunks * p.batch > INT32_MAX) return RPX_ERR_SHAPE;
    return launch_on_top(tree_join_kernel<D, Cut, kSplit, kJoinRows>, static_cast<unsigned>(chunks * p.batch), kJoinWarps * 32, 0, stream, p,
                         static_cast<int32_t>(chunks));
}
// More than 8 pieces per segment: a block a row.  Else 32 rows a warp (tensor-core form), or a row, or where there are more
// rows than the SMs hold warps, two (streaming form, whole call with a row and with two: 200 rows 15.3 and 15.7 us, 5120 rows
// 38.2 and 38.9, 7680 rows 52.9 and 52.1, 12288 rows 78.6 and 77.1).
template <int D, int kTiles>
rpx_status_t launch_join_tiles(const Params& p, cudaStream_t stream) {
    using Cut = NodeCut<kTiles>;
    const int32_t blocks = Cut::blocks(p, p.max_tree);
    const int64_t segments = static_cast<int64_t>(p.batch) * p.num_kv_heads * blocks, grid = segments * (Cut::kRows / 32 * (D / 32) / kJoinWarps);
    if (p.ctas > 8 * segments) return launch_join_split<D, Cut, kJoinWarps, 1>(p, stream);
    if (grid > INT32_MAX) return RPX_ERR_SHAPE;
    return launch_on_top(tree_join_tiles_kernel<D, kTiles>, static_cast<unsigned>(grid), kJoinWarps * 32, 0, stream, p, blocks);
}
template <int D, class Cut>
rpx_status_t launch_join_rows(const Params& p, cudaStream_t stream) {
    const int64_t segments = static_cast<int64_t>(p.batch) * p.num_kv_heads * Cut::blocks(p, p.max_tree);
    if (p.ctas > 8 * segments) return launch_join_split<D, Cut, kJoinWarps, 1>(p, stream);
    return p.total_tokens * p.num_q_heads > 6144 ? launch_join_split<D, Cut, 1, 2>(p, stream) : launch_join_split<D, Cut, 1, 1>(p, stream);
}

// The pass's workspace: sequences' first units, then the pieces' rows.
template <class Cut>
inline size_t join_workspace(int32_t batch, int32_t ctas, int32_t head_dim) {
    const size_t rows = static_cast<size_t>(ctas) * 2 * Cut::kRows;
    return align_up(static_cast<size_t>(batch + 1) * sizeof(int64_t), 256) + align_up(rows * sizeof(float2), 256) + rows * head_dim * sizeof(float);
}
template <class Cut>
inline void carve_workspace(Params& p, void* workspace) {
    uint8_t* ws = static_cast<uint8_t*>(workspace);
    p.seq_unit0 = reinterpret_cast<int64_t*>(ws);
    ws += align_up(static_cast<size_t>(p.batch + 1) * sizeof(int64_t), 256);
    p.part_ml = reinterpret_cast<float2*>(ws);
    ws += align_up(static_cast<size_t>(p.ctas) * 2 * Cut::kRows * sizeof(float2), 256);
    p.part_o = reinterpret_cast<float*>(ws);
}

// Short sequences are not cut: one CTA walks a segment of up to kWholeTiles key tiles in less time than cutting and joining
// take (head_dim 128; 4 x 1 nodes, streaming: 300 cached tokens 9.5 us whole and 10.3 cut, 400: 11.1 and 9.5; 2 x 16 nodes,
// one query tile: 900 tokens 19.2 and 20.8, 1100: 20.2 and 20.7; 2 x 100 nodes, two: 700 tokens 22.6 and 24.2, 1100: 28.0 and
// 24.6.  head_dim 64, in the same order: 7.5 and 8.8, 8.6 and 8.3; 17.4 and 18.8, 18.4 and 18.9; 19.5 and 20.9, 24.2 and 21.0).
// Goes by the caller's bound; a longer sequence is only slower.  Returns the grid (and sets whole_blocks), or 0.
template <class Cut>
inline int64_t whole_grid(Params& p, int32_t max_cached) {
    const int64_t tiles = (static_cast<int64_t>(max_cached) + Cut::kTile - 1) / Cut::kTile + (p.max_tree + Cut::kTile - 1) / Cut::kTile;
    const int32_t blocks = Cut::blocks(p, p.max_tree);
    const int64_t grid = static_cast<int64_t>(p.batch) * p.num_kv_heads * blocks;
    if (tiles > Cut::kWholeTiles || grid > INT32_MAX) return 0;
    p.whole_blocks = blocks;
    return grid;
}

inline Params make_params(const TreeArgs& a) {
    Params p = {};
    p.q = static_cast<const __nv_bfloat16*>(a.q);
    p.q_stride = a.q_tok_stride;
    p.cu = a.cu_seqlens;
    p.parents = a.parents;
    p.lens = a.cached_lens;
    p.block_table = a.cache->block_table;
    p.block_table_stride = a.cache->block_table_stride;
    p.num_blocks = static_cast<int32_t>(a.cache->num_blocks);
    p.k_cache = static_cast<const __nv_bfloat16*>(a.cache->k_cache);
    p.v_cache = static_cast<const __nv_bfloat16*>(a.cache->v_cache);
    p.batch = a.batch;
    p.num_q_heads = a.num_q_heads;
    p.num_kv_heads = a.num_kv_heads;
    p.group = a.num_q_heads / a.num_kv_heads;
    p.tile_nodes = p.group <= 128 ? 128 / p.group : 1;
    p.max_tree = a.max_tree;
    p.total_tokens = a.total_tokens;
    const float scale = a.softmax_scale > 0.f ? a.softmax_scale : 1.0f / sqrtf(static_cast<float>(a.head_dim));
    p.scale_log2 = scale * kLog2e;
    p.out = static_cast<__nv_bfloat16*>(a.out);
    p.lse = a.lse;
    p.status = a.device_status;
    return p;
}

}  // namespace tree
}  // namespace rpx
