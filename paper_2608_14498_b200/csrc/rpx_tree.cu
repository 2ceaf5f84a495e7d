// Attention of a tree of drafted tokens over [cached prefix ; ancestors in the tree], for few rows: the streaming form.
//
// For node i of a sequence, query head h and KV head g = h / group, over the cached keys 0 .. len - 1 and the nodes j on
// the path from i to its root (i included):   out = sum_j softmax_j(scale * q . k_j) v_j.
//
// With few nodes (one is a decoding step) this is bound by reading the cache: every cached K and V is read once per block of
// up to 64 rows (row = node * group + head within the KV head's group), 512 bytes per key against rows * 512 flops.  So
// the work is laid out along the keys (rpx_tree.cuh): a single long sequence spreads over all SMs as evenly as a ragged
// batch does.
//   warp 4     : producer; one TMA box per 16-token page and tensor (both 64-element halves of its rows in one box,
//                128-byte swizzle), three stages of 64 keys of K and V
//   warps 0-3  : S = Q K^T and O += P V with mma.sync (16 rows x 8 keys x 16): at these row counts the tensor rate is not
//                what bounds, and a 16-row tile wastes least of it.  A block is 16, 32 or 64 rows; the four warps are
//                kRowTiles row tiles x 4 / kRowTiles ranges of the tile's keys, and join their ranges in shared memory
//                at the end of a segment.
// Scores are kept in log2 units, the running maximum is raised lazily (by steps of at least 2^8), sums are fp32.
#include "rpx_tree.cuh"

namespace rpx {

namespace {

using namespace tree;

constexpr int kTile = 64, kStages = 3;
constexpr int kWarps = 4;  // consumer warps
constexpr int kThreads = 32 * (kWarps + 1);
constexpr int kCtasPerSm = 2;
constexpr int kMaxNodes = 128;   // nodes per sequence this form takes (their ancestor sets live in shared memory)
constexpr int kMaskWords = kMaxNodes / 32;

struct Ctl {
    uint64_t full[kStages], empty[kStages];
    uint32_t issued;  // tiles the producer has asked for
    uint32_t abort_flag, drain_flag, data_error;
    float2 ml[kWarps][16];
    uint32_t anc[kMaxNodes][kMaskWords];  // ancestors and itself; all zero for a node that is not in use
};

template <int D>
struct Layout {
    static constexpr int kPageBytes = kPage * D * 2;
    static constexpr int kTensorBytes = kTile * D * 2;
    static constexpr int kStageBytes = 2 * kTensorBytes;
    static constexpr int kCtlOff = kStages * kStageBytes;
    static constexpr size_t kSmemBytes = kCtlOff + sizeof(Ctl);
};

// shared-memory offset of 16-byte chunk c of key r within a tile: pages of [half][16 rows][128 bytes], swizzled
template <int D>
__device__ __forceinline__ uint32_t key_off(int r, int c) {
    return (r >> 4) * Layout<D>::kPageBytes + (c >> 3) * (kPage * 128) + (r & 15) * 128 + (((c & 7) ^ (r & 7)) << 4);
}

__device__ __forceinline__ void consumer_sync() { asm volatile("bar.sync 1, 128;" ::: "memory"); }

template <int D, int kRowTiles>
__global__ void __launch_bounds__(kThreads, kCtasPerSm)
tree_stream_kernel(const __grid_constant__ CUtensorMap tmap_k, const __grid_constant__ CUtensorMap tmap_v,
                   const __grid_constant__ CUtensorMap tmap_kc, const __grid_constant__ CUtensorMap tmap_vc, const Params p) {
    using L = Layout<D>;
    constexpr int kRows = 16 * kRowTiles;
    using Cut = RowCut<kRows>;
    constexpr int kRanges = kWarps / kRowTiles;  // key ranges of a tile the warps work on side by side
    constexpr int kSteps = kTile / kRanges / 16; // 16-key steps of one range
    extern __shared__ __align__(1024) uint8_t smem[];
    if ((smem_u32(smem) & 1023u) != 0u) {  // swizzled pages need 1024-byte alignment; never expected
        if (threadIdx.x == 0 && p.status != nullptr) atomicCAS(p.status, 0, RPX_ERR_CUDA);
        return;
    }
    Ctl* ctl = reinterpret_cast<Ctl*>(smem + L::kCtlOff);
    volatile uint32_t* abort_flag = &ctl->abort_flag;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (threadIdx.x == 0) {
        for (int i = 0; i < kStages; ++i) {
            mbar_init(&ctl->full[i], 1);
            mbar_init(&ctl->empty[i], kWarps);
        }
        ctl->abort_flag = ctl->drain_flag = ctl->data_error = 0;
        ctl->issued = 0;
        fence_barrier_init();
    }
    __syncthreads();
    Walk<Cut> walk(p, find_piece<Cut>(p, &ctl->data_error));
    uint32_t it = 0;  // tiles this warp has been through (ring position)
    bool ok = true;

    if (warp == kWarps) {
        // =========================================================== producer
        while (ok && walk.next(p)) {
            const int32_t pg = lane & 3;
            const int32_t* table = p.block_table + static_cast<int64_t>(walk.s) * p.block_table_stride;
            const int32_t pages = (walk.q.len + kPage - 1) / kPage;
            auto read_block = [&](int32_t t) { return t * 4 + pg < pages ? __ldg(table + t * 4 + pg) : 0; };
            int32_t next_block = walk.t0 < walk.q.cached_tiles ? read_block(walk.t0) : 0;
            for (int32_t t = walk.t0; t < walk.t1; ++t, ++it) {
                const uint32_t st = it % kStages;
                if (!mbar_wait(&ctl->empty[st], ((it / kStages) & 1u) ^ 1u, abort_flag)) {
                    ok = false;
                    break;
                }
                uint8_t* dst = smem + st * L::kStageBytes + (lane >> 2) * L::kTensorBytes + pg * L::kPageBytes;
                const bool cached = t < walk.q.cached_tiles;
                int32_t block = next_block;
                const int32_t own = t - walk.q.cached_tiles;  // the tree's own tile number
                const int32_t boxes = cached ? min(4, pages - t * 4) : min(4, (walk.q.n - own * kTile + kPage - 1) / kPage);
                if (cached) {
                    if (block < 0 || block >= p.num_blocks) {
                        ctl->data_error = 1;
                        block = 0;
                    }
                    if (t + 1 < walk.q.cached_tiles && t + 1 < walk.t1) next_block = read_block(t + 1);
                }
                if (lane == 0) mbar_arrive_expect_tx(&ctl->full[st], static_cast<uint32_t>(boxes) * 2 * L::kPageBytes);
                __syncwarp();  // the byte count is armed before any copy can complete
                if (lane < 8 && pg < boxes) {  // lanes 0-3: the pages of K, lanes 4-7: those of V
                    if (cached) tma_load_5d(dst, lane < 4 ? &tmap_kc : &tmap_vc, &ctl->full[st], 0, 0, 0, walk.head, block);
                    else tma_load_4d(dst, lane < 4 ? &tmap_k : &tmap_v, &ctl->full[st], 0, walk.q.tok0 + own * kTile + pg * kPage, 0, walk.head);
                }
                __syncwarp();
            }
        }
        if (lane == 0) ctl->issued = it;
        asm volatile("griddepcontrol.launch_dependents;" ::: "memory");  // every load is on its way: the join may start soon
    } else {
        // =========================================================== consumers
        // After a wait that ran out (ok == false) a warp goes through the rest of its walk without waiting: every warp
        // still meets the others at the same barriers, and the outputs of the call are undefined anyway.
        const int rt = warp % kRowTiles, range = warp / kRowTiles;
        const int gid = lane >> 2, tid = lane & 3;
        while (walk.next(p)) {
            const Seq q = walk.q;
            const int32_t rows = q.n * p.group, row0 = walk.block * kRows;
            // ---- Q of the warp's 16 rows, as A operands
            uint32_t qf[D / 16][4];
            int32_t node[2];
            {
                const __nv_bfloat16* src[2];
                bool there[2];
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    const int32_t r = row0 + rt * 16 + gid + 8 * u;
                    there[u] = r < rows;
                    node[u] = there[u] ? r / p.group : 0;
                    src[u] = p.q + (static_cast<int64_t>(q.tok0) + node[u]) * p.q_stride +
                             (static_cast<int64_t>(walk.head) * p.group + (there[u] ? r - node[u] * p.group : 0)) * D + 2 * tid;
                }
#pragma unroll
                for (int ks = 0; ks < D / 16; ++ks)
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        qf[ks][e] = there[e & 1] ? __ldg(reinterpret_cast<const uint32_t*>(src[e & 1] + ks * 16 + 8 * (e >> 1))) : 0u;
            }
            // ---- the tree's ancestor sets, where this piece reaches its keys
            const bool has_own = walk.t1 > q.cached_tiles;
            if (has_own) {
                for (int32_t j = threadIdx.x; j < q.n; j += 32 * kWarps) {
                    uint32_t bits[kMaskWords];
#pragma unroll
                    for (int w = 0; w < kMaskWords; ++w) bits[w] = 0u;
                    int32_t at = j;
                    bool good = true, used = true;
                    while (at >= 0) {
#pragma unroll
                        for (int w = 0; w < kMaskWords; ++w)
                            if (w == (at >> 5)) bits[w] |= 1u << (at & 31);
                        const int32_t up = __ldg(p.parents + q.tok0 + at);
                        if (up < -1 && at == j) used = false;          // padding
                        else if (up < -1 || up >= at) good = false;    // hangs on padding, or on a later node
                        if (up >= at) break;
                        at = up;
                    }
                    if (!good) ctl->data_error = 1;
#pragma unroll
                    for (int w = 0; w < kMaskWords; ++w) ctl->anc[j][w] = good && used ? bits[w] : 0u;
                }
                consumer_sync();
            }
            // Probabilities are rounded to bf16 for the P V product.  Over few keys that rounding is not averaged away, so
            // short segments carry P as two bf16 terms (2^-17).
            const bool two_terms = kRowTiles <= 2 || q.tiles <= 4;
            float o[D / 8][4];
#pragma unroll
            for (int i = 0; i < D / 8; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e) o[i][e] = 0.f;
            float run_max[2] = {-CUDART_INF_F, -CUDART_INF_F}, run_sum[2] = {0.f, 0.f};

            for (int32_t t = walk.t0; t < walk.t1; ++t, ++it) {
                const uint32_t st = it % kStages;
                if (ok) ok = mbar_wait(&ctl->full[st], (it / kStages) & 1u, abort_flag);
                uint8_t* stage = smem + st * L::kStageBytes;
                const uint32_t k_addr = smem_u32(stage), v_addr = k_addr + L::kTensorBytes;
                const bool own = t >= q.cached_tiles;
                const int32_t first = (own ? t - q.cached_tiles : t) * kTile;  // number of the tile's first key
                const int32_t keys = min(kTile, (own ? q.n : q.len) - first);  // keys the tile holds
                // V rows behind the last key, and those of unused nodes, may hold anything: a probability of 0 must not
                // meet a NaN there, so they are cleared (up to the next 16-key step; steps beyond it are not computed)
                const bool clear = own || (keys & 15) != 0;
                if (clear) {
                    const int32_t r = threadIdx.x >> 1;
                    if (r < ((keys + 15) & ~15) &&
                        (r >= keys || (own && ((ctl->anc[first + r][(first + r) >> 5] >> ((first + r) & 31)) & 1u) == 0u))) {
#pragma unroll
                        for (int c = 0; c < D / 16; ++c)
                            *reinterpret_cast<uint4*>(stage + L::kTensorBytes + key_off<D>(r, (threadIdx.x & 1) * (D / 16) + c)) =
                                make_uint4(0u, 0u, 0u, 0u);
                    }
                    consumer_sync();
                }
                // ---- scores of the warp's 16 rows and its range's keys
                const int32_t range0 = range * kSteps * 16;
                if (range0 < keys) {
                    float sc[2 * kSteps][4];
#pragma unroll
                    for (int j = 0; j < kSteps; ++j) {
                        const int32_t k0 = range0 + j * 16;
                        if (k0 >= keys) {
#pragma unroll
                            for (int e = 0; e < 4; ++e) sc[2 * j][e] = sc[2 * j + 1][e] = -CUDART_INF_F;
                            continue;
                        }
#pragma unroll
                        for (int e = 0; e < 4; ++e) sc[2 * j][e] = sc[2 * j + 1][e] = 0.f;
                        const int32_t r = k0 + (lane & 7) + ((lane >> 4) << 3);
#pragma unroll
                        for (int ks = 0; ks < D / 16; ++ks) {
                            uint32_t b[4];
                            ldsm_x4(k_addr + key_off<D>(r, 2 * ks + ((lane >> 3) & 1)), b);
                            mma_16x8x16(sc[2 * j], qf[ks], b[0], b[1]);
                            mma_16x8x16(sc[2 * j + 1], qf[ks], b[2], b[3]);
                        }
                    }
                    if (own) {
#pragma unroll
                        for (int i = 0; i < 2 * kSteps; ++i)
#pragma unroll
                            for (int e = 0; e < 4; ++e) {
                                const int32_t j = first + range0 + 8 * i + 2 * tid + (e & 1);
                                if (j >= q.n || ((ctl->anc[node[e >> 1]][j >> 5] >> (j & 31)) & 1u) == 0u) sc[i][e] = -CUDART_INF_F;
                            }
                    } else if (keys < kTile) {
#pragma unroll
                        for (int i = 0; i < 2 * kSteps; ++i)
#pragma unroll
                            for (int e = 0; e < 4; ++e)
                                if (range0 + 8 * i + 2 * tid + (e & 1) >= keys) sc[i][e] = -CUDART_INF_F;
                    }
                    // ---- online softmax; a row is spread over four lanes
                    float alpha[2], base[2];
                    bool grow = false;
#pragma unroll
                    for (int u = 0; u < 2; ++u) {
                        float m = fmaxf(sc[0][2 * u], sc[0][2 * u + 1]);
#pragma unroll
                        for (int i = 1; i < 2 * kSteps; ++i) m = fmaxf(m, fmaxf(sc[i][2 * u], sc[i][2 * u + 1]));
                        m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 1));
                        m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 2)) * p.scale_log2;
                        const bool up = m > run_max[u] + kRaise;
                        const float to = up ? m : run_max[u];
                        alpha[u] = up ? fast_exp2(run_max[u] - to) : 1.f;
                        grow |= up;
                        run_max[u] = to;
                        base[u] = to == -CUDART_INF_F ? 0.f : to;  // a row that has seen no key yet
                        run_sum[u] *= alpha[u];
                    }
                    if (__any_sync(0xffffffffu, grow)) {
#pragma unroll
                        for (int i = 0; i < D / 8; ++i)
#pragma unroll
                            for (int e = 0; e < 4; ++e) o[i][e] *= alpha[e >> 1];
                    }
#pragma unroll
                    for (int j = 0; j < kSteps; ++j) {
                        const int32_t k0 = range0 + j * 16;
                        if (k0 >= keys) break;
                        uint32_t hi[4], lo[4];
#pragma unroll
                        for (int e = 0; e < 4; ++e) {  // operand word e: row half e & 1, key half e >> 1
                            const int i = 2 * j + (e >> 1), u = e & 1;
                            const float x = fast_exp2(fmaf(sc[i][2 * u], p.scale_log2, -base[u]));
                            const float y = fast_exp2(fmaf(sc[i][2 * u + 1], p.scale_log2, -base[u]));
                            run_sum[u] += x + y;
                            hi[e] = pack_bf16x2(x, y);
                            lo[e] = pack_bf16x2(x - __uint_as_float(hi[e] << 16), y - __uint_as_float(hi[e] & 0xffff0000u));
                        }
                        const int32_t r = k0 + (lane & 15);
#pragma unroll
                        for (int dp = 0; dp < D / 16; ++dp) {
                            uint32_t b[4];
                            ldsm_x4_trans(v_addr + key_off<D>(r, 2 * dp + (lane >> 4)), b);
                            mma_16x8x16(o[2 * dp], hi, b[0], b[1]);
                            mma_16x8x16(o[2 * dp + 1], hi, b[2], b[3]);
                            if (two_terms) {
                                mma_16x8x16(o[2 * dp], lo, b[0], b[1]);
                                mma_16x8x16(o[2 * dp + 1], lo, b[2], b[3]);
                            }
                        }
                    }
                }
                if (t + 1 < walk.t1) {  // the last tile's stage first serves the join below
                    if (clear) fence_proxy_async_smem();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&ctl->empty[st]);
                }
            }
            // ---- join the warps' key ranges in the last tile's stage and hand the rows on
            const uint32_t last = (it - 1) % kStages;
            float* joined = reinterpret_cast<float*>(smem + last * L::kStageBytes);  // [warp][16][D]: as large as the stage
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                run_sum[u] += __shfl_xor_sync(0xffffffffu, run_sum[u], 1);
                run_sum[u] += __shfl_xor_sync(0xffffffffu, run_sum[u], 2);
                if (tid == 0) ctl->ml[warp][gid + 8 * u] = make_float2(run_max[u], run_sum[u]);
            }
            consumer_sync();  // nobody reads the tile any more
#pragma unroll
            for (int i = 0; i < D / 8; ++i)
#pragma unroll
                for (int u = 0; u < 2; ++u)  // columns xor 8 * (row % 8): the eight rows of a store hit different banks
                    *reinterpret_cast<float2*>(joined + (warp * 16 + gid + 8 * u) * D + ((8 * i + 2 * tid) ^ (gid << 3))) =
                        make_float2(o[i][2 * u], o[i][2 * u + 1]);
            consumer_sync();
            const bool whole = walk.t0 == 0 && walk.t1 == q.tiles;
            const int64_t slot = (static_cast<int64_t>(blockIdx.x) * 2 + (walk.t0 == 0 ? 1 : 0)) * kRows;
            for (int32_t i = threadIdx.x; i < kRows * (D / 4); i += 32 * kWarps) {
                const int32_t r = i / (D / 4), c = (i % (D / 4)) * 4, rr = r & 15;
                if (row0 + r >= rows) break;
                float top = -CUDART_INF_F;
#pragma unroll
                for (int w = 0; w < kRanges; ++w) top = fmaxf(top, ctl->ml[(r >> 4) + w * kRowTiles][rr].x);
                float sum = 0.f;
                float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
                for (int w = 0; w < kRanges; ++w) {
                    const float2 ml = ctl->ml[(r >> 4) + w * kRowTiles][rr];
                    // a range that saw no key contributes nothing (and its maximum is no number to subtract)
                    const float f = ml.x == -CUDART_INF_F ? 0.f : fast_exp2(ml.x - top);
                    const float4 v = *reinterpret_cast<const float4*>(joined + (((r >> 4) + w * kRowTiles) * 16 + rr) * D + (c ^ ((rr & 7) << 3)));
                    sum = fmaf(f, ml.y, sum);
                    acc.x = fmaf(f, v.x, acc.x);
                    acc.y = fmaf(f, v.y, acc.y);
                    acc.z = fmaf(f, v.z, acc.z);
                    acc.w = fmaf(f, v.w, acc.w);
                }
                const int32_t nd = (row0 + r) / p.group;
                // a piece that reaches the tree's own keys knows whether the row's node is in use
                const bool unused = walk.t1 == q.tiles && ((ctl->anc[nd][nd >> 5] >> (nd & 31)) & 1u) == 0u;
                if (whole) {
                    const int64_t row = (static_cast<int64_t>(q.tok0) + nd) * p.num_q_heads + walk.head * p.group + (row0 + r - nd * p.group);
                    const float inv = unused ? 0.f : 1.f / sum;
                    uint2 w;
                    w.x = unused ? 0u : pack_bf16x2(acc.x * inv, acc.y * inv);
                    w.y = unused ? 0u : pack_bf16x2(acc.z * inv, acc.w * inv);
                    *reinterpret_cast<uint2*>(p.out + row * D + c) = w;
                    if (c == 0 && p.lse != nullptr) p.lse[row] = unused ? -CUDART_INF_F : (top + log2f(sum)) * kLn2;
                } else {
                    *reinterpret_cast<float4*>(p.part_o + (slot + r) * D + c) = acc;
                    if (c == 0) p.part_ml[slot + r] = make_float2(top, unused ? -1.f : sum);  // a negative sum marks an unused node
                }
            }
            fence_proxy_async_smem();  // plain stores to the stage, before the next copy into it
            consumer_sync();
            if (lane == 0) mbar_arrive(&ctl->empty[last]);
        }
    }
    __syncthreads();
    if (threadIdx.x == 0 && ctl->abort_flag != 0u) {  // copies still in flight get a moment to land before the memory is released
        const uint32_t n = ctl->issued, first = n > kStages ? n - kStages : 0u;
        for (uint32_t i = first; i < n; ++i)
            mbar_wait(&ctl->full[i % kStages], (i / kStages) & 1u, &ctl->drain_flag, kDrainLimitCycles);
    }
    if (threadIdx.x == 0 && p.status != nullptr) {
        if (ctl->abort_flag != 0u) atomicCAS(p.status, 0, RPX_ERR_TIMEOUT);
        else if (ctl->data_error != 0u) atomicCAS(p.status, 0, RPX_ERR_DEVICE_DATA);
    }
}

constexpr int kMaxCtas = 148 * kCtasPerSm;  // the workspace is sized for this many pieces

// Rows per block: the smallest of 16, 32 and 64 that holds a tree's rows of one KV head.
int rows_per_block(int64_t rows) { return rows <= 16 ? 16 : rows <= 32 ? 32 : 64; }

template <int D, int kRowTiles>
rpx_status_t launch_stream(const TreeArgs& a, const CUtensorMap& tk, const CUtensorMap& tv, const CUtensorMap& tkc,
                           const CUtensorMap& tvc, Params p) {
    using L = Layout<D>;
    using Cut = RowCut<16 * kRowTiles>;
    auto* kernel = tree_stream_kernel<D, kRowTiles>;
    if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(L::kSmemBytes)) != cudaSuccess)
        return RPX_ERR_CUDA;
    carve_workspace<Cut>(p, a.workspace);
    const int64_t whole = whole_grid<Cut>(p, a.max_cached);
    kernel<<<static_cast<unsigned>(whole > 0 ? whole : p.ctas), kThreads, L::kSmemBytes, a.stream>>>(tk, tv, tkc, tvc, p);
    if (cudaGetLastError() != cudaSuccess) return RPX_ERR_CUDA;
    if (whole > 0) return RPX_OK;
    return launch_join_rows<D, Cut>(p, a.stream);
}

template <int D>
rpx_status_t launch_stream_d(const TreeArgs& a) {
    CUtensorMap tk, tv, tkc, tvc;
    {
        // the tree's own K, V: 16 tokens of one head as a page: (64 elements, token, half, head)
        const uint64_t dims[4] = {64, static_cast<uint64_t>(a.total_tokens), D / 64, static_cast<uint64_t>(a.num_kv_heads)};
        const uint64_t ks[3] = {static_cast<uint64_t>(a.k_tok_stride) * 2, 128, D * 2ull};
        const uint64_t vs[3] = {static_cast<uint64_t>(a.v_tok_stride) * 2, 128, D * 2ull};
        const uint32_t box[4] = {64, kPage, D / 64, 1};
        if (rpx_status_t rc = encode_tmap_bf16(&tk, a.k, 4, dims, ks, box)) return rc;
        if (rpx_status_t rc = encode_tmap_bf16(&tv, a.v, 4, dims, vs, box)) return rc;
    }
    {
        const uint64_t dims[5] = {64, kPage, D / 64, static_cast<uint64_t>(a.num_kv_heads), static_cast<uint64_t>(a.cache->num_blocks)};
        const uint64_t strides[4] = {D * 2ull, 128, kPage * D * 2ull, static_cast<uint64_t>(a.num_kv_heads) * kPage * D * 2ull};
        const uint32_t box[5] = {64, kPage, D / 64, 1, 1};
        if (rpx_status_t rc = encode_tmap_bf16(&tkc, a.cache->k_cache, 5, dims, strides, box)) return rc;
        if (rpx_status_t rc = encode_tmap_bf16(&tvc, a.cache->v_cache, 5, dims, strides, box)) return rc;
    }
    Params p = make_params(a);
    const int sms = sm_count();
    if (sms <= 0) return RPX_ERR_CUDA;
    // (the SM budget is left out of this: where the line of tiles is cut decides the order of the sums, and this pass does
    // not hold an SM for longer than its share of one read of the cache)
    p.ctas = sms * kCtasPerSm < kMaxCtas ? sms * kCtasPerSm : kMaxCtas;
    switch (rows_per_block(static_cast<int64_t>(a.max_tree) * p.group)) {
        case 16: return launch_stream<D, 1>(a, tk, tv, tkc, tvc, p);
        case 32: return launch_stream<D, 2>(a, tk, tv, tkc, tvc, p);
        default: return launch_stream<D, 4>(a, tk, tv, tkc, tvc, p);
    }
}

// ------------------------------------------------------------------ ancestor sets and values for the other forms
// One warp per token: its ancestor set as mask words (lane w holds word w while all lanes walk the path to the root), all
// zero for a node that is not in use or a token of no sequence; and, for the tensor-core form, a copy of the
// tree's V with those rows cleared (a probability of 0 must not meet what they hold), 8 rows more for every sequence before it
// and zeros behind its last node: what is copied 8 rows at a time then never holds another sequence's values.
constexpr int kSetWarps = 8;
__global__ void __launch_bounds__(kSetWarps * 32)
tree_sets_kernel(const int32_t* __restrict__ cu, const int32_t* __restrict__ parents, int32_t batch, int64_t total_tokens,
                 int32_t max_tree, int32_t words, uint32_t* sets, const __nv_bfloat16* v, int64_t v_stride, int32_t v_chunks,
                 __nv_bfloat16* v_copy, int32_t* status) {
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");  // the attention kernel may start on its cached tiles
    // Parents of the sequence that the block's first token is in: the walk is a chain of dependent reads (192 nodes in
    // steps of three: 10 us from global memory, which kept the attention kernel off the SMs).
    __shared__ int32_t staged[RPX_TREE_MAX_NODES];
    const int lane = threadIdx.x & 31;
    const int64_t first = static_cast<int64_t>(blockIdx.x) * kSetWarps, token = first + (threadIdx.x >> 5);
    auto sequence_of = [&](int64_t t) {  // the last that starts at or before the token
        int32_t lo = 0, hi = batch - 1;
        while (lo < hi) {
            const int32_t mid = (lo + hi + 1) >> 1;
            if (__ldg(cu + mid) <= t) lo = mid;
            else hi = mid - 1;
        }
        return lo;
    };
    auto inside_of = [&](int64_t t, int32_t begin, int64_t n) {
        return begin >= 0 && begin <= t && t < begin + n && begin + n <= total_tokens && n <= max_tree;
    };
    const int32_t s0 = sequence_of(first), begin0 = __ldg(cu + s0);
    const int64_t n0 = static_cast<int64_t>(__ldg(cu + s0 + 1)) - begin0;
    if (inside_of(first, begin0, n0))
        for (int32_t i = threadIdx.x; i < n0; i += kSetWarps * 32) staged[i] = __ldg(parents + begin0 + i);
    __syncthreads();
    if (token >= total_tokens) return;
    int32_t tok0 = begin0, s = s0;
    int64_t n = n0;
    if (token >= begin0 + n0) {
        s = sequence_of(token);
        tok0 = __ldg(cu + s);
        n = static_cast<int64_t>(__ldg(cu + s + 1)) - tok0;
    }
    const bool inside = inside_of(token, tok0, n), is_staged = tok0 == begin0 && n == n0 && inside_of(first, begin0, n0);
    uint32_t bits = 0u;
    bool good = true, used = inside;
    int32_t at = inside ? static_cast<int32_t>(token - tok0) : -1;
    const int32_t self = at;
    while (at >= 0) {
        if ((at >> 5) == lane) bits |= 1u << (at & 31);
        const int32_t up = is_staged ? staged[at] : __ldg(parents + tok0 + at);
        if (up < -1 && at == self) used = false;
        else if (up < -1 || up >= at) good = false;
        if (up >= at) break;
        at = up;
    }
    if (!good && lane == 0 && status != nullptr) atomicCAS(status, 0, RPX_ERR_DEVICE_DATA);
    used = used && good;
    if (lane < words) sets[token * words + lane] = used ? bits : 0u;
    if (v_copy != nullptr && inside) {
        const uint4* src = reinterpret_cast<const uint4*>(v + token * v_stride);
        uint4* dst = reinterpret_cast<uint4*>(v_copy) + (token + 8ll * s) * v_chunks;
        for (int32_t i = lane; i < v_chunks; i += 32) dst[i] = used ? __ldg(src + i) : make_uint4(0u, 0u, 0u, 0u);
        if (token == tok0 + n - 1)  // zeros up to the next 8 rows of the sequence
            for (int32_t i = lane; i < static_cast<int32_t>(-n & 7) * v_chunks; i += 32) dst[v_chunks + i] = make_uint4(0u, 0u, 0u, 0u);
    }
}

}  // namespace

int32_t tree_set_words(int32_t max_tree) { return (max_tree + 127) / 128 * 4; }

rpx_status_t launch_tree_sets(const TreeArgs& a, uint32_t* sets, void* v_copy) {
    const int64_t blocks = (a.total_tokens + kSetWarps - 1) / kSetWarps;
    tree_sets_kernel<<<static_cast<unsigned>(blocks), kSetWarps * 32, 0, a.stream>>>(
        a.cu_seqlens, a.parents, a.batch, a.total_tokens, a.max_tree, tree_set_words(a.max_tree), sets,
        static_cast<const __nv_bfloat16*>(a.v), a.v_tok_stride, a.num_kv_heads * a.head_dim / 8,
        static_cast<__nv_bfloat16*>(v_copy), a.device_status);
    return cudaGetLastError() == cudaSuccess ? RPX_OK : RPX_ERR_CUDA;
}

// The streaming form reads the cache at 95 % of the copy rate with one row tile (32 x 3 nodes of 5 heads over 8192 tokens: 173
// us) and 82 % with two (32 x 6 nodes: 200 us); with four, mma.sync bounds it, and the tensor-core form is faster at every
// length (2 x 8 nodes of 7 heads over 600 tokens 17 us against 35, 8 x 16 over 1000 22 against 32).  That one takes trees of
// any size, but groups of at most 128 heads.
bool tree_streams(int32_t max_tree, int32_t group) {
    return max_tree <= kMaxNodes && (static_cast<int64_t>(max_tree) * group <= 32 || group > 128);
}

size_t tree_stream_workspace(int32_t batch, int32_t head_dim) { return join_workspace<RowCut<64>>(batch, kMaxCtas, head_dim); }

rpx_status_t launch_tree_stream(const TreeArgs& a) {
    return a.head_dim == 128 ? launch_stream_d<128>(a) : launch_stream_d<64>(a);
}

}  // namespace rpx
