// Attention of a tree of drafted tokens over [cached prefix ; ancestors in the tree], for many rows: the tensor-core form.
//
// Same mathematics and the same cut as the streaming form (rpx_tree.cuh), with 128-key tiles and tcgen05.  A query tile is
// tile_nodes = 128 / group nodes times the query heads of one KV head (row = node * group + head), so a key tile is
// fetched once for all of them.  A block holds one query tile, or two where trees need more rows (kPaired).  Per 128 keys
// a query tile costs 1024 clocks of tensor pipe, 1024 of exponentials, and the tile itself 64 KB, 1.48 us (2500 clocks) of this
// SM's share of HBM: with one query tile the cache's bytes bound, provided that the softmax of one step hides behind the
// products of another.  So there are always two score buffers in flight:
//   two query tiles  the buffers are the query tiles, both walk every key tile;
//   one query tile   the buffers take turns: buffer t walks the key tiles t, t + 2, .. with a running maximum, sum and
//                    output of its own, and both buffers' warps add the two up straight out of TMEM at the end.
// Measured by a fit over the CTAs (head_dim 128): a key tile against one query tile 1.35 us where the bytes bound it and 1.0
// where they come from L2, against two 1.67 us, going over to another segment 4.5 - 6.5 us.  Of the 3200 clocks of a tile
// against two, the tensor core is busy for 2050, and its issuer waits 1200 for probabilities and 800 for K and V; handing the
// probabilities over in two halves, or waiting for K behind the first product instead of in front of it, changed nothing.
//   warps 0-3, 4-7 : softmax of buffer 0, 1: thread = row = TMEM lane
//   warp  8        : producer: Q once per segment, K and V through rings of their own (K runs a tile ahead, so it is not
//                    held up behind a V slot), one TMA box per 16-token page
//   warp  9        : issues S_t = Q K^T (smem x smem -> TMEM) and O_t += P_t V (P as bf16 over S_t's first 64 columns)
//   warps 10, 11   : only take part in the register hand-over
// The tree's own V tiles come from a copy in which rows of unused nodes are zero (and no other sequence's rows follow), and
// ancestor sets as bit masks; a small kernel writes both (tree_sets_kernel).  This kernel is launched on top of that one and
// waits for it only where it first needs its results, behind the cached tiles.
#include <type_traits>

#include "rpx_tree.cuh"

namespace rpx {

namespace {

using namespace tree;

constexpr int kTile = 128, kPages = kTile / kPage;
constexpr int kThreads = 32 * 12;
constexpr int kProducerWarp = 8, kMmaWarp = 9;
constexpr int kSoftmaxRegs = 208, kOtherRegs = 88;  // 256 * 208 + 128 * 88 <= 384 * 168, what the launch has
constexpr uint32_t kTmemCols = 512;
constexpr int kMaxCtas = 148;

template <int D, bool kPaired>
struct Layout {
    static constexpr int kHalves = D / 64;
    static constexpr int kHalfBytes = kTile * 128;  // one [128 rows][64 bf16] swizzled block
    static constexpr int kTensorBytes = kHalves * kHalfBytes;
    static constexpr int kQTiles = kPaired ? 2 : 1;
    static constexpr int kSlotsK = 3, kSlotsV = kPaired ? 2 : 3;
    static constexpr int kKOff = kQTiles * kTensorBytes;
    static constexpr int kVOff = kKOff + kSlotsK * kTensorBytes;
    static constexpr int kCtlOff = kVOff + kSlotsV * kTensorBytes;
};

struct Ctl {
    uint64_t q_full, q_empty;
    uint64_t k_full[3], k_empty[3], v_full[3], v_empty[3];
    uint64_t s_full[2];   // tensor core -> softmax: the scores of a step (and the product before it has read its P)
    uint64_t p_ready[2];  // softmax -> tensor core
    uint64_t o_done[2];   // tensor core -> softmax: the segment's last product into O_t
    uint64_t o_free[2];   // softmax -> tensor core: O_t has been read
    uint64_t ml_ready;    // both buffers' maxima and sums are in `ml`
    uint64_t drain;
    uint32_t tmem_base, abort_flag, drain_flag, data_error;
    float2 ml[2][kTile];
    int32_t walk[8][20];  // the softmax warps' walks: in registers they spill, and local memory is hundreds of clocks away
    int32_t more[8];
};

// Key tiles lie as [group of 8 keys][half][8 rows][128 bytes], swizzled: a 16-token page (two groups, both halves) is one
// 4 KB TMA box, and to the tensor core the groups are evenly spaced, which is all that its descriptors need.  (With a box
// per page and half, 32 boxes of 2 KB a tile, the loads took 3800 clocks per 64 KB tile whatever the pass did with them.)
template <int D>
__device__ __forceinline__ uint32_t key_off(int r, int c) {  // of 16-byte chunk c of key r
    return static_cast<uint32_t>(((r >> 3) * (D / 64) + (c >> 3)) * 1024 + (r & 7) * 128 + (((c & 7) ^ (r & 7)) << 4));
}

// Waits until the kernel launched before this one has finished and its writes are visible.
__device__ __forceinline__ void wait_for_sets() { asm volatile("griddepcontrol.wait;" ::: "memory"); }

template <int D, bool kPaired>
__global__ void __launch_bounds__(kThreads, 1)
tree_tile_kernel(const __grid_constant__ CUtensorMap tmap_q, const __grid_constant__ CUtensorMap tmap_k,
                 const __grid_constant__ CUtensorMap tmap_v, const __grid_constant__ CUtensorMap tmap_kc,
                 const __grid_constant__ CUtensorMap tmap_vc, const Params p) {
    using L = Layout<D, kPaired>;
    using Cut = NodeCut<L::kQTiles>;
    extern __shared__ __align__(1024) uint8_t smem[];
    if ((smem_u32(smem) & 1023u) != 0u) {  // swizzled tiles need 1024-byte alignment; never expected
        if (threadIdx.x == 0 && p.status != nullptr) atomicCAS(p.status, 0, RPX_ERR_CUDA);
        return;
    }
    Ctl* ctl = reinterpret_cast<Ctl*>(smem + L::kCtlOff);
    volatile uint32_t* abort_flag = &ctl->abort_flag;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (threadIdx.x == 0) {
        mbar_init(&ctl->q_full, 1);
        mbar_init(&ctl->q_empty, 1);
        for (int i = 0; i < 3; ++i) {
            mbar_init(&ctl->k_full[i], 1);
            mbar_init(&ctl->k_empty[i], 1);
            mbar_init(&ctl->v_full[i], 1);
            mbar_init(&ctl->v_empty[i], 1);
        }
        for (int t = 0; t < 2; ++t) {
            mbar_init(&ctl->s_full[t], 1);
            mbar_init(&ctl->p_ready[t], 4);
            mbar_init(&ctl->o_done[t], 1);
            mbar_init(&ctl->o_free[t], 8);
        }
        mbar_init(&ctl->ml_ready, 8);
        mbar_init(&ctl->drain, 1);
        ctl->abort_flag = ctl->drain_flag = ctl->data_error = 0;
        fence_barrier_init();
    }
    if (warp == kMmaWarp) {
        tmem_alloc(&ctl->tmem_base, kTmemCols);
        tmem_relinquish();
    }
    tc_fence_before_sync();
    __syncthreads();
    tc_fence_after_sync();
    const uint32_t tmem_base = ctl->tmem_base;  // S_t at columns 128 t, O_t at 256 + 128 t
    const Piece piece = find_piece<Cut>(p, &ctl->data_error);
    // Every role walks the piece's segments alike.  A block whose nodes fit one query tile lets the buffers take turns.
    auto nodes_in_block = [&](const Walk<Cut>& walk) { return min(walk.q.n - walk.block * L::kQTiles * p.tile_nodes, L::kQTiles * p.tile_nodes); };

    if (warp == kProducerWarp) {
        // =========================================================== producer
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kOtherRegs));
        Walk<Cut> walk(p, piece);
        bool ok = true, have_sets = false;
        uint32_t nk = 0, nv = 0, segments = 0;
        while (ok && walk.next(p)) {
            const Seq q = walk.q;
            const int32_t node0 = walk.block * L::kQTiles * p.tile_nodes;
            const bool paired = kPaired && nodes_in_block(walk) > p.tile_nodes;
            if (segments > 0 && !mbar_wait(&ctl->q_empty, (segments - 1) & 1u, abort_flag)) {
                ok = false;
                break;
            }
            if (lane == 0) {  // one box of tile_nodes nodes x group heads lands as consecutive 128-byte rows
                mbar_arrive_expect_tx(&ctl->q_full, (paired ? 2 : 1) * L::kHalves * p.tile_nodes * p.group * 128);
                for (int t = 0; t < (paired ? 2 : 1); ++t)
                    for (int hf = 0; hf < L::kHalves; ++hf)
                        tma_load_3d(smem + t * L::kTensorBytes + hf * L::kHalfBytes, &tmap_q, &ctl->q_full, hf * 64,
                                    walk.head * p.group, q.tok0 + node0 + t * p.tile_nodes);
            }
            ++segments;
            const int32_t* table = p.block_table + static_cast<int64_t>(walk.s) * p.block_table_stride;
            const int32_t pages = (q.len + kPage - 1) / kPage;
            // lane pg fetches page pg of a tile; block ids are read a tile ahead and looked at only then
            const int pg = lane & 7;
            auto read_block = [&](int32_t t) { return t < q.cached_tiles && t * kPages + pg < pages ? __ldg(table + t * kPages + pg) : 0; };
            auto load = [&](int32_t t, int32_t block, bool is_v, uint8_t* dst, uint64_t* full) {
                if (t >= q.cached_tiles) {  // the tree's own keys
                    const int32_t own = t - q.cached_tiles;
                    if (is_v && !have_sets) {
                        wait_for_sets();
                        have_sets = true;
                    }
                    const int32_t boxes = min(kTile / 8, (q.n - own * kTile + 7) / 8);  // tokens start anywhere: a box per 8
                    if (is_v && boxes < kTile / 8) {  // zeros behind the tree's last rows (what K holds there is masked)
                        for (int32_t i = lane; i < (kTile - boxes * 8) * (D / 8); i += 32)
                            *reinterpret_cast<uint4*>(dst + key_off<D>(boxes * 8 + i / (D / 8), i % (D / 8))) = make_uint4(0u, 0u, 0u, 0u);
                        fence_proxy_async_smem();
                        __syncwarp();
                    }
                    if (lane == 0) mbar_arrive_expect_tx(full, boxes * 8 * D * 2);
                    __syncwarp();
                    if (lane < boxes)
                        tma_load_4d(dst + lane * (8 * D * 2), is_v ? &tmap_v : &tmap_k, full, 0,
                                    q.tok0 + own * kTile + lane * 8 + (is_v ? 8 * walk.s : 0), 0, walk.head);
                    return;
                }
                // K behind the last key may be anything (its scores are masked); V may not: what a probability of 0 meets
                // is the ragged page's rows up to the last key, copied by hand, and zeros
                const int32_t rows = min(kTile, q.len - t * kTile);
                const int32_t boxes = is_v ? rows / kPage : (rows + kPage - 1) / kPage;
                if (is_v && boxes < kPages) {
                    const int32_t ragged = __shfl_sync(0xffffffffu, block, boxes);
                    const uint4* src = reinterpret_cast<const uint4*>(p.v_cache + (static_cast<int64_t>(ragged) * p.num_kv_heads + walk.head) * kPage * D);
                    const int32_t first = boxes * kPage;
                    uint4 x[kPage * D / 8 / 32];
#pragma unroll
                    for (int i = 0; i < kPage * D / 8 / 32; ++i) {  // the page, all loads in flight together
                        const int32_t r = (lane + 32 * i) / (D / 8);
                        x[i] = make_uint4(0u, 0u, 0u, 0u);
                        if (first + r < rows) x[i] = __ldg(src + lane + 32 * i);
                    }
#pragma unroll
                    for (int i = 0; i < kPage * D / 8 / 32; ++i)
                        *reinterpret_cast<uint4*>(dst + key_off<D>(first + (lane + 32 * i) / (D / 8), (lane + 32 * i) % (D / 8))) = x[i];
                    for (int32_t i = lane; i < (kTile - first - kPage) * (D / 8); i += 32)
                        *reinterpret_cast<uint4*>(dst + key_off<D>(first + kPage + i / (D / 8), i % (D / 8))) = make_uint4(0u, 0u, 0u, 0u);
                    fence_proxy_async_smem();
                    __syncwarp();
                }
                if (lane == 0) {
                    if (boxes > 0) mbar_arrive_expect_tx(full, boxes * kPage * D * 2);
                    else mbar_arrive(full);
                }
                __syncwarp();  // the byte count is armed before any copy can complete
                if (lane < boxes)
                    tma_load_4d(dst + pg * (kPage * D * 2), is_v ? &tmap_vc : &tmap_kc, full, 0, 0, 0, (block * p.num_kv_heads + walk.head) * 2);
            };
            const int32_t n = walk.t1 - walk.t0;
            int32_t block_now = read_block(walk.t0), block_before = 0;
            for (int32_t j = 0; ok && j <= n; ++j) {
                const int32_t block_next = j + 1 < n ? read_block(walk.t0 + j + 1) : 0;
                if (j < n) {
                    const uint32_t st = nk % L::kSlotsK;
                    ok = mbar_wait(&ctl->k_empty[st], ((nk / L::kSlotsK) & 1u) ^ 1u, abort_flag);
                    if (!ok) break;
                    if (block_now < 0 || block_now >= p.num_blocks) {
                        ctl->data_error = 1;
                        block_now = 0;
                    }
                    load(walk.t0 + j, block_now, false, smem + L::kKOff + st * L::kTensorBytes, &ctl->k_full[st]);
                    ++nk;
                    __syncwarp();
                }
                if (j > 0) {
                    const uint32_t st = nv % L::kSlotsV;
                    ok = mbar_wait(&ctl->v_empty[st], ((nv / L::kSlotsV) & 1u) ^ 1u, abort_flag);
                    if (!ok) break;
                    load(walk.t0 + j - 1, block_before, true, smem + L::kVOff + st * L::kTensorBytes, &ctl->v_full[st]);
                    ++nv;
                    __syncwarp();
                }
                block_before = block_now;
                block_now = block_next;
            }
        }
        if (!ok) {  // abort: copies still in flight get a moment to land before shared memory is released
            for (uint32_t i = nk > L::kSlotsK ? nk - L::kSlotsK : 0u; i < nk; ++i)
                mbar_wait(&ctl->k_full[i % L::kSlotsK], (i / L::kSlotsK) & 1u, &ctl->drain_flag, kDrainLimitCycles);
            for (uint32_t i = nv > L::kSlotsV ? nv - L::kSlotsV : 0u; i < nv; ++i)
                mbar_wait(&ctl->v_full[i % L::kSlotsV], (i / L::kSlotsV) & 1u, &ctl->drain_flag, kDrainLimitCycles);
            if (segments > 0) mbar_wait(&ctl->q_full, (segments - 1) & 1u, &ctl->drain_flag, kDrainLimitCycles);
        }
    } else if (warp == kMmaWarp) {
        // =========================================================== tcgen05 issuer (one thread)
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kOtherRegs));
        if (elect_one()) {
            Walk<Cut> walk(p, piece);
            constexpr uint32_t idesc_qk = make_idesc_bf16(kTile, kTile, false, false);
            constexpr uint32_t idesc_pv = make_idesc_bf16(kTile, D, false, true);
            const uint64_t q_desc = make_smem_desc_sw128(smem_u32(smem), 16, 1024);
            const uint64_t k_desc = make_smem_desc_sw128(smem_u32(smem + L::kKOff), 16, L::kHalves * 1024);    // K-major
            const uint64_t v_desc = make_smem_desc_sw128(smem_u32(smem + L::kVOff), 1024, L::kHalves * 1024);  // MN-major
            bool ok = true;
            uint32_t segments = 0, nk = 0, nv = 0;
            uint32_t steps[2] = {0, 0};  // steps of each buffer so far (barrier parity)
            uint32_t used[2] = {0, 0};   // segments in which it took part
            auto wait_k = [&](uint32_t i) { return mbar_wait(&ctl->k_full[i % L::kSlotsK], (i / L::kSlotsK) & 1u, abort_flag); };
            auto wait_v = [&](uint32_t i) { return mbar_wait(&ctl->v_full[i % L::kSlotsV], (i / L::kSlotsV) & 1u, abort_flag); };
            auto issue_qk = [&](int t, int tile, uint32_t i) {
                const uint64_t kd = k_desc + static_cast<uint64_t>((i % L::kSlotsK) * (L::kTensorBytes >> 4));
                const uint64_t qd = q_desc + static_cast<uint64_t>(tile * (L::kTensorBytes >> 4));
#pragma unroll
                for (int ks = 0; ks < D / 16; ++ks)  // 16 columns = 32 bytes of a 128-byte row
                    umma_bf16_ss(tmem_base + t * 128, qd + (ks >> 2) * (L::kHalfBytes >> 4) + 2 * (ks & 3), kd + (ks >> 2) * 64 + 2 * (ks & 3),
                                 idesc_qk, ks != 0);
                umma_commit(&ctl->s_full[t]);
            };
            // waits for the probabilities of a buffer's next step and issues their product with V
            auto issue_pv = [&](int t, uint32_t i, bool first, bool two_terms) {
                if (!mbar_wait(&ctl->p_ready[t], steps[t] & 1u, abort_flag)) return false;
                ++steps[t];
                // the first product of a segment overwrites O_t: the one before must have been read
                if (first && used[t] > 0 && !mbar_wait(&ctl->o_free[t], (used[t] - 1) & 1u, abort_flag)) return false;
                tc_fence_after_sync();
                const uint64_t vd = v_desc + static_cast<uint64_t>((i % L::kSlotsV) * (L::kTensorBytes >> 4));
#pragma unroll
                for (int ks = 0; ks < kTile / 16; ++ks)  // 16 keys = 8 columns of P = two groups of V
                    umma_bf16_ts(tmem_base + 256 + t * 128, tmem_base + t * 128 + 8 * ks, vd + ks * (L::kHalves * 128), idesc_pv, !first || ks != 0);
                if (two_terms)
#pragma unroll
                    for (int ks = 0; ks < kTile / 16; ++ks)
                        umma_bf16_ts(tmem_base + 256 + t * 128, tmem_base + t * 128 + 64 + 8 * ks, vd + ks * (L::kHalves * 128), idesc_pv, 1u);
                return true;
            };
            while (ok && walk.next(p)) {
                const int32_t n = walk.t1 - walk.t0;
                const bool paired = kPaired && nodes_in_block(walk) > p.tile_nodes;
                const bool two_terms = walk.q.tiles <= 2;
                ok = mbar_wait(&ctl->q_full, segments & 1u, abort_flag);
                if (paired) {
                    if (ok) ok = wait_k(nk);
                    if (!ok) break;
                    tc_fence_after_sync();
                    issue_qk(0, 0, nk);
                    issue_qk(1, 1, nk);
                    umma_commit(&ctl->k_empty[nk % L::kSlotsK]);
                    if (n == 1) umma_commit(&ctl->q_empty);
                    for (int32_t j = 0; ok && j < n; ++j) {
                        const bool more = j + 1 < n;
                        if (!wait_v(nv + j) || (more && !wait_k(nk + j + 1))) {
                            ok = false;
                            break;
                        }
                        for (int t = 0; ok && t < 2; ++t) {
                            ok = issue_pv(t, nv + j, j == 0, two_terms);
                            if (!ok) break;
                            if (more) issue_qk(t, t, nk + j + 1);  // in order behind the product: P_t is read before S_t is rewritten
                            else umma_commit(&ctl->o_done[t]);
                        }
                        if (!ok) break;
                        umma_commit(&ctl->v_empty[(nv + j) % L::kSlotsV]);
                        if (more) umma_commit(&ctl->k_empty[(nk + j + 1) % L::kSlotsK]);
                        if (j == n - 2) umma_commit(&ctl->q_empty);
                    }
                    if (!ok) break;
                    ++used[0];
                    ++used[1];
                } else {
                    for (int32_t j = 0; ok && j < min(n, 2); ++j) {
                        ok = wait_k(nk + j);
                        if (!ok) break;
                        tc_fence_after_sync();
                        issue_qk(j, 0, nk + j);
                        umma_commit(&ctl->k_empty[(nk + j) % L::kSlotsK]);
                    }
                    if (!ok) break;
                    if (n <= 2) umma_commit(&ctl->q_empty);
                    for (int32_t j = 0; j < n; ++j) {
                        const int t = j & 1;
                        ok = wait_v(nv + j) && issue_pv(t, nv + j, j < 2, two_terms);
                        if (!ok) break;
                        umma_commit(&ctl->v_empty[(nv + j) % L::kSlotsV]);
                        if (j + 2 < n) {
                            ok = wait_k(nk + j + 2);
                            if (!ok) break;
                            tc_fence_after_sync();
                            issue_qk(t, 0, nk + j + 2);
                            umma_commit(&ctl->k_empty[(nk + j + 2) % L::kSlotsK]);
                            if (j + 3 == n) umma_commit(&ctl->q_empty);
                        } else {
                            umma_commit(&ctl->o_done[t]);
                        }
                    }
                    if (!ok) break;
                    ++used[0];
                    if (n > 1) ++used[1];
                }
                nk += n;
                nv += n;
                ++segments;
            }
            if (!ok) {
                umma_commit(&ctl->drain);
                mbar_wait(&ctl->drain, 0, &ctl->drain_flag, kDrainLimitCycles);
            }
        }
        __syncwarp();
        // What is left is the last segment's output: once every CTA is there, the join may start on the SMs that are free.
        // (Earlier, and it would crowd the SMs that finish first.)
        asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    } else if (warp > kMmaWarp) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kOtherRegs));
    } else {
        // =========================================================== softmax
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kSoftmaxRegs));
        const int t = warp >> 2;
        const int32_t row = (warp & 3) * 32 + lane;
        const uint32_t lane_addr = static_cast<uint32_t>((warp & 3) * 32) << 16;
        const uint32_t my_s = tmem_base + t * 128 + lane_addr, my_o = tmem_base + 256 + t * 128 + lane_addr;
        uint32_t steps = 0;              // this buffer's steps so far
        uint32_t used[2] = {0, 0};       // segments in which each buffer took part
        uint32_t turns = 0;              // segments in which the buffers took turns
        bool ok = true, have_sets = false;
        static_assert(sizeof(Walk<Cut>) <= sizeof(ctl->walk[0]), "room for a walk");
        Walk<Cut>& walk = *reinterpret_cast<Walk<Cut>*>(ctl->walk[warp]);
        if (lane == 0) walk = Walk<Cut>(p, piece);
        while (ok) {
            __syncwarp();  // the segment before has been read
            if (lane == 0) ctl->more[warp] = walk.next(p) ? 1 : 0;
            __syncwarp();
            if (ctl->more[warp] == 0) break;
            const int32_t tok0 = walk.q.tok0, len = walk.q.len, cached_tiles = walk.q.cached_tiles, t0 = walk.t0, n = walk.t1 - walk.t0;
            const bool has_last = walk.t1 == walk.q.tiles, whole = has_last && t0 == 0;
            const bool paired = kPaired && nodes_in_block(walk) > p.tile_nodes;
            const bool two_terms = walk.q.tiles <= 2;
            const int32_t in_tile = row / p.group;  // rows beyond tile_nodes * group are padding
            const int32_t node = walk.block * L::kQTiles * p.tile_nodes + (paired ? t * p.tile_nodes : 0) + in_tile;
            const bool row_valid = in_tile < p.tile_nodes && node < walk.q.n;
            const int32_t head = walk.head * p.group + (row - in_tile * p.group);
            // ---- ancestor set, where this piece reaches the tree's own keys
            const uint32_t* set = nullptr;
            uint32_t own_word = ~0u;  // holds the node's own bit; looked at by the pieces with the last tile, one of the tree's own
            if (t0 + n > cached_tiles) {
                if (!have_sets) {
                    wait_for_sets();
                    have_sets = true;
                }
                if (row_valid) {
                    set = p.sets + (static_cast<int64_t>(tok0) + node) * p.set_words;
                    own_word = set[node >> 5];
                }
            }
            float run_max = -CUDART_INF_F, run_sum = 0.f;
            bool first = true;
            // instantiated twice, so that the usual form keeps its registers
            auto run_steps = [&](auto two_terms_tag) {
            constexpr bool kTwoTerms = decltype(two_terms_tag)::value;
            for (int32_t j = paired ? 0 : t; j < n; j += paired ? 1 : 2) {
                if (!mbar_wait(&ctl->s_full[t], steps & 1u, abort_flag)) {
                    ok = false;
                    break;
                }
                ++steps;
                tc_fence_after_sync();
                uint32_t sc[4][32];
#pragma unroll
                for (int c = 0; c < 4; ++c) tmem_ld32(my_s + c * 32, sc[c]);
                tmem_ld_wait();
                const int32_t tile = t0 + j;
                if (tile >= cached_tiles) {
                    uint4 m = make_uint4(0u, 0u, 0u, 0u);
                    if (set != nullptr) m = reinterpret_cast<const uint4*>(set)[tile - cached_tiles];
                    const uint32_t bits[4] = {m.x, m.y, m.z, m.w};
#pragma unroll
                    for (int c = 0; c < 4; ++c)
#pragma unroll
                        for (int i = 0; i < 32; ++i)
                            if (((bits[c] >> i) & 1u) == 0u) sc[c][i] = 0xff800000u;  // -inf
                } else if (len - tile * kTile < kTile) {
                    const int32_t keys = len - tile * kTile;
#pragma unroll
                    for (int c = 0; c < 4; ++c)
#pragma unroll
                        for (int i = 0; i < 32; ++i)
                            if (c * 32 + i >= keys) sc[c][i] = 0xff800000u;
                }
                auto score = [&](int e) { return __uint_as_float(sc[e >> 5][e & 31]); };
                float mx[8];
#pragma unroll
                for (int u = 0; u < 8; ++u) mx[u] = fmax3(score(u), score(8 + u), score(16 + u));
#pragma unroll
                for (int e = 24; e < kTile - 8; e += 16)
#pragma unroll
                    for (int u = 0; u < 8; ++u) mx[u] = fmax3(mx[u], score(e + u), score(e + 8 + u));
#pragma unroll
                for (int u = 0; u < 4; ++u) mx[u] = fmax3(mx[u], score(kTile - 8 + u), score(kTile - 4 + u));
                const float m = fmax3(fmax3(mx[0], mx[1], mx[2]), fmax3(mx[3], mx[4], mx[5]), fmax3(mx[6], mx[7], mx[7])) * p.scale_log2;
                const bool grow = m > run_max + kRaise;
                const float new_max = grow ? m : run_max;
                const float alpha = grow ? fast_exp2(run_max - new_max) : 1.f;
                const bool rescale = !first && __any_sync(0xffffffffu, grow);
                run_sum *= alpha;
                run_max = new_max;
                const float base = run_max == -CUDART_INF_F ? 0.f : run_max;  // a row that has seen no key yet
                // ---- P = 2^(x - max): bf16 pairs over the first 64 columns of S_t, for short segments (one or two tiles,
                // where the rounding is not averaged over many keys) a second term in the other 64.  All exponentials go to the
                // special-function unit: 0 for a masked key (-inf), NaN for NaN and for +inf (inf - inf).  With a quarter of them
                // as a polynomial on the FMA pipe, clamped at 2^-125, a masked key had that weight, which a value of 1e38 shows,
                // and the pass was no faster (8 x 8 nodes 27.8 us against 26.5, 32 ragged trees 212 against 207.5, 8 x 192 the same).
                const uint64_t scale2 = f2_pack(p.scale_log2, p.scale_log2), base2 = f2_pack(-base, -base);
                uint64_t part[4] = {0ull, 0ull, 0ull, 0ull};
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    uint32_t packed[16];
                    [[maybe_unused]] uint32_t lo[4];
#pragma unroll
                    for (int i = 0; i < 32; i += 2) {
                        float x0, x1;
                        f2_unpack(f2_fma(f2_pack(__uint_as_float(sc[c][i]), __uint_as_float(sc[c][i + 1])), scale2, base2), x0, x1);
                        const float e0 = fast_exp2(x0), e1 = fast_exp2(x1);
                        part[(i / 2) % 4] = f2_add(part[(i / 2) % 4], f2_pack(e0, e1));
                        packed[i >> 1] = pack_bf16x2(e0, e1);
                        if constexpr (kTwoTerms) {  // what the first term dropped
                            lo[(i >> 1) & 3] = pack_bf16x2(e0 - __uint_as_float(packed[i >> 1] << 16), e1 - __uint_as_float(packed[i >> 1] & 0xffff0000u));
                            if (((i >> 1) & 3) == 3) tmem_st4(my_s + 64 + c * 16 + (i >> 1) - 3, lo);
                        }
                    }
                    tmem_st16(my_s + c * 16, packed);
                }
                {
                    float a0, a1;
                    f2_unpack(f2_add(f2_add(part[0], part[1]), f2_add(part[2], part[3])), a0, a1);
                    run_sum += a0 + a1;
                }
                // the scores of this step were committed behind the product before it, so O_t is quiet until the arrival below
                if (rescale) {
#pragma unroll 1
                    for (int c = 0; c < D / 32; ++c) {
                        uint32_t r[32];
                        tmem_ld32(my_o + c * 32, r);
                        tmem_ld_wait();
#pragma unroll
                        for (int i = 0; i < 32; ++i) r[i] = __float_as_uint(__uint_as_float(r[i]) * alpha);
                        tmem_st32(my_o + c * 32, r);
                    }
                }
                first = false;
                tmem_st_wait();
                tc_fence_before_sync();
                __syncwarp();
                if (lane == 0) mbar_arrive(&ctl->p_ready[t]);
            }
            };
            if (two_terms) run_steps(std::true_type{});
            else run_steps(std::false_type{});
            if (!ok) break;
            // ---- the segment's rows.  Two query tiles: each buffer's warps write their own.  One: the warps of both buffers
            // add the two outputs up, one half of the columns each.
            const bool with_1 = paired || n > 1;  // buffer 1 took part
            float f0 = 1.f, f1 = 0.f, top = run_max, sum = run_sum;
            if (paired) {
                ok = mbar_wait(&ctl->o_done[t], used[t] & 1u, abort_flag);
            } else {
                // (whoever has let go of O_0 has read the maxima and sums of the segment before)
                ok = used[0] == 0 || mbar_wait(&ctl->o_free[0], (used[0] - 1) & 1u, abort_flag);
                if (!ok) break;
                ctl->ml[t][row] = make_float2(run_max, run_sum);
                __syncwarp();
                if (lane == 0) mbar_arrive(&ctl->ml_ready);
                ok = mbar_wait(&ctl->ml_ready, turns & 1u, abort_flag) && mbar_wait(&ctl->o_done[0], used[0] & 1u, abort_flag) &&
                     (!with_1 || mbar_wait(&ctl->o_done[1], used[1] & 1u, abort_flag));
                ++turns;
                if (ok) {
                    const float2 a = ctl->ml[0][row], b = ctl->ml[1][row];
                    top = fmaxf(a.x, b.x);
                    f0 = a.x == -CUDART_INF_F ? 0.f : fast_exp2(a.x - top);
                    f1 = b.x == -CUDART_INF_F ? 0.f : fast_exp2(b.x - top);
                    sum = f0 * a.y + f1 * b.y;
                }
            }
            if (!ok) break;
            tc_fence_after_sync();
            ++used[0];
            if (with_1) ++used[1];
            const bool adds = !paired && with_1;
            const uint32_t o_addr = tmem_base + 256 + (paired ? t * 128 : 0) + lane_addr;
            const int c_begin = paired || t == 0 ? 0 : D / 64, c_end = paired || t == 1 ? D / 32 : D / 64;
            const bool unused = has_last && ((own_word >> (node & 31)) & 1u) == 0u;
            const int64_t out_row = (static_cast<int64_t>(tok0) + node) * p.num_q_heads + head;
            const int64_t slot = (static_cast<int64_t>(blockIdx.x) * 2 + (t0 == 0 ? 1 : 0)) * Cut::kRows + (paired ? t * 128 : 0) + row;
            const float inv = top == -CUDART_INF_F ? CUDART_NAN_F : 1.f / sum;  // (every score -inf: 0 / 0)
            const bool wide = (reinterpret_cast<uintptr_t>(p.out) & 31u) == 0u;
#pragma unroll 1
            for (int c = c_begin; c < c_end; ++c) {
                uint32_t a[32], b[32];
                tmem_ld32(o_addr + c * 32, a);
                if (adds) tmem_ld32(o_addr + 128 + c * 32, b);
                tmem_ld_wait();
                if (c == c_end - 1) {  // O is out of TMEM: the next segment's first product may overwrite it
                    tc_fence_before_sync();
                    __syncwarp();
                    if (lane == 0) {  // eight arrivals: four warps twice, or all eight
                        if (paired) {
                            mbar_arrive(&ctl->o_free[t]);
                            mbar_arrive(&ctl->o_free[t]);
                        } else {
                            mbar_arrive(&ctl->o_free[0]);
                            if (adds) mbar_arrive(&ctl->o_free[1]);
                        }
                    }
                }
                if (adds) {
#pragma unroll
                    for (int i = 0; i < 32; ++i)
                        a[i] = __float_as_uint(fmaf(f0, __uint_as_float(a[i]), f1 * __uint_as_float(b[i])));
                }
                if (!whole) {  // (rows that are padding go along: they are nobody's)
                    float* dst = p.part_o + Cut::template part_at<D>(slot, c * 32);
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        st_global_v8(dst + 256 * i, a[8 * i], a[8 * i + 1], a[8 * i + 2], a[8 * i + 3], a[8 * i + 4], a[8 * i + 5],
                                     a[8 * i + 6], a[8 * i + 7]);
                } else if (row_valid) {
                    uint32_t w[16];
#pragma unroll
                    for (int i = 0; i < 16; ++i)
                        w[i] = unused ? 0u : pack_bf16x2(__uint_as_float(a[2 * i]) * inv, __uint_as_float(a[2 * i + 1]) * inv);
                    __nv_bfloat16* dst = p.out + out_row * D + c * 32;
                    if (wide) {
                        st_global_v8(dst, w[0], w[1], w[2], w[3], w[4], w[5], w[6], w[7]);
                        st_global_v8(dst + 16, w[8], w[9], w[10], w[11], w[12], w[13], w[14], w[15]);
                    } else {
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            reinterpret_cast<uint4*>(dst)[i] = make_uint4(w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]);
                    }
                }
            }
            if (row_valid && (paired || t == 0)) {
                if (!whole) p.part_ml[slot] = make_float2(top, unused ? -1.f : sum);
                else if (p.lse != nullptr) p.lse[out_row] = unused ? -CUDART_INF_F : (top + log2f(sum)) * kLn2;
            }
        }
    }

    tc_fence_before_sync();
    __syncthreads();
    if (warp == kMmaWarp) {
        tc_fence_after_sync();
        tmem_dealloc(tmem_base, kTmemCols);
    }
    wait_for_sets();  // this kernel never ends before the one it was launched on top of
    if (threadIdx.x == 0 && p.status != nullptr) {
        if (ctl->abort_flag != 0u) atomicCAS(p.status, 0, RPX_ERR_TIMEOUT);
        else if (ctl->data_error != 0u) atomicCAS(p.status, 0, RPX_ERR_DEVICE_DATA);
    }
}

template <int D, bool kPaired>
rpx_status_t launch_tile(const TreeArgs& a, const uint32_t* sets, const void* values) {
    using L = Layout<D, kPaired>;
    using Cut = NodeCut<L::kQTiles>;
    Params p = make_params(a);
    p.sets = sets;
    p.set_words = tree_set_words(a.max_tree);
    const int sms = sm_count();
    if (sms <= 0) return RPX_ERR_CUDA;
    p.ctas = sms < kMaxCtas ? sms : kMaxCtas;  // (without the SM budget: see the streaming form)
    carve_workspace<Cut>(p, a.workspace);
    CUtensorMap tq, tk, tv, tkc, tvc;
    const uint64_t tokens = static_cast<uint64_t>(a.total_tokens), heads = static_cast<uint64_t>(a.num_kv_heads);
    {
        const uint64_t dims[3] = {D, static_cast<uint64_t>(a.num_q_heads), tokens};
        const uint64_t strides[2] = {D * 2ull, static_cast<uint64_t>(a.q_tok_stride) * 2};
        const uint32_t box[3] = {64, static_cast<uint32_t>(p.group), static_cast<uint32_t>(p.tile_nodes)};
        if (rpx_status_t rc = encode_tmap_bf16(&tq, a.q, 3, dims, strides, box)) return rc;
    }
    {
        const uint64_t dims[4] = {64, tokens, D / 64, heads}, vdims[4] = {64, tokens + 8ull * a.batch, D / 64, heads};
        const uint64_t ks[3] = {static_cast<uint64_t>(a.k_tok_stride) * 2, 128, D * 2ull}, vs[3] = {heads * D * 2ull, 128, D * 2ull};
        const uint32_t box[4] = {64, 8, D / 64, 1};
        if (rpx_status_t rc = encode_tmap_bf16(&tk, a.k, 4, dims, ks, box)) return rc;
        if (rpx_status_t rc = encode_tmap_bf16(&tv, values, 4, vdims, vs, box)) return rc;
    }
    {
        // the pool as groups of 8 keys: two per page and head
        const uint64_t groups = static_cast<uint64_t>(a.cache->num_blocks) * heads * 2;  // (fits 32 bits: checked by the caller)
        const uint64_t dims[4] = {64, 8, D / 64, groups};
        const uint64_t strides[3] = {D * 2ull, 128, 8 * D * 2ull};
        const uint32_t box[4] = {64, 8, D / 64, 2};
        if (rpx_status_t rc = encode_tmap_bf16(&tkc, a.cache->k_cache, 4, dims, strides, box)) return rc;
        if (rpx_status_t rc = encode_tmap_bf16(&tvc, a.cache->v_cache, 4, dims, strides, box)) return rc;
    }
    constexpr size_t smem = L::kCtlOff + sizeof(Ctl);
    static_assert(smem <= 232448, "shared memory of one CTA");
    auto* kernel = tree_tile_kernel<D, kPaired>;
    if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(smem)) != cudaSuccess) return RPX_ERR_CUDA;
    const int64_t whole = whole_grid<Cut>(p, a.max_cached);
    if (rpx_status_t rc = launch_on_top(kernel, static_cast<unsigned>(whole > 0 ? whole : p.ctas), kThreads, smem, a.stream, tq, tk, tv, tkc, tvc, p))
        return rc;
    if (whole > 0) return RPX_OK;
    return launch_join_tiles<D, L::kQTiles>(p, a.stream);
}

// One query tile holds the rows of every tree: the buffers take turns throughout and the second Q tile's room goes to V.
bool paired(int32_t max_tree, int32_t group) { return max_tree > 128 / group; }

}  // namespace

size_t tree_tile_workspace(int32_t batch, int32_t head_dim, int32_t max_tree, int32_t group) {
    return paired(max_tree, group) ? join_workspace<NodeCut<2>>(batch, kMaxCtas, head_dim) : join_workspace<NodeCut<1>>(batch, kMaxCtas, head_dim);
}

rpx_status_t launch_tree_tile(const TreeArgs& a, const uint32_t* sets, const void* values) {
    if (paired(a.max_tree, a.num_q_heads / a.num_kv_heads))
        return a.head_dim == 128 ? launch_tile<128, true>(a, sets, values) : launch_tile<64, true>(a, sets, values);
    return a.head_dim == 128 ? launch_tile<128, false>(a, sets, values) : launch_tile<64, false>(a, sets, values);
}

}  // namespace rpx
