// Attention of groups of sequences over the paged cache: the kernel that walks the key tiles (bf16).
//
// Few query rows meet many keys here - 5 to 8 rows a sequence in a decoding step, some dozens where a group shares a prompt -
// and every cached byte is read once, 512 bytes a key against rows * 512 flops.  So the KEYS are the tensor core's M: a key
// tile's 128 keys are the 128 lanes of S^T = K Q^T, the rows are its columns, and what a tile costs grows with the rows that are
// there (16 to 64 in steps of 16) instead of with a tile of 128 that holds them:
//     S^T [128 keys x N rows]  = K [128 x D] (K-major, as it lies in the cache) * Q^T (K-major)
//     O^T [D x N rows]        += V^T [D x 128] (V as it lies in the cache, read MN-major) * P^T [128 x N]
// P goes through shared memory, as bf16 [row][key] (K-major B operand).  The scores are loaded from tensor memory in the fragment
// that stmatrix takes (16 lanes x 256 bits: a thread holds two rows of one key), so a warp stores its 32 keys of eight rows
// with one instruction.  Half of P's room takes what the rounding to bf16 dropped, as so many more rows of the same product:
// probabilities enter it as two terms (off by 2^-17) and not as one (2^-8), and the two outputs are added when they are read.  That
// costs nothing where the cache's bytes bound: V, the larger operand, is read once.  (Blocks of 112 rows with one term took 102 us
// where blocks of 64 with both take 130, 4 prompts of 64 responses, and were off by 0.0023 of the largest output for 0.0017.)
//
// A row's running reference is raised only when a score passes it by 2^8: what is kept is exact whatever the reference, so all
// the threads of a tile need to agree on is whether one of them has to (one barrier with a vote).
//
// Segments (a KV head's keys of a group's prompt or of one sequence) follow one another without a pause: there are two buffers
// each of S, P, O and Q, every product has a thread of its own that waits for its own operands only, and
// a segment's output is written by warps that do nothing else, while the softmax warps are in the next one.
//   4 x 2 or 4 warps : two (up to 16 rows) or four teams with a share of the rows each: softmax, lanes = keys
//   1 warp each      : producer of K and V (one TMA box per 16-token page); S^T = K Q^T; O^T += V^T P^T; laying Q out
//   4 warps          : output, lanes = elements of D

#include "rpx_group.cuh"

namespace rpx {

namespace {

using namespace group;

constexpr int kPages = kTile / kPage;
constexpr float kRaise = 8.0f;  // log2 units
constexpr int kMaxSlots = 6;

template <int D, int kCap>
struct Layout {
    static constexpr int kTeams = kCap == 16 ? 2 : 4;              // of four softmax warps
    static constexpr int kProducerWarp = 4 * kTeams, kScoreWarp = kProducerWarp + 1, kValueWarp = kProducerWarp + 2, kQWarp = kProducerWarp + 3;
    static constexpr int kOutWarp = kProducerWarp + 4;             // the first of four
    static constexpr int kThreads = 32 * (kOutWarp + 4);
    static constexpr int kBlocks = (kCap / 8 + kTeams - 1) / kTeams;  // 8-row blocks of a team at most
    static constexpr int kHalves = D / 64;
    static constexpr int kTensorBytes = kTile * D * 2;             // a key tile of K or V
    static constexpr int kPRows = 2 * kCap;                        // of both terms
    static constexpr int kPHalfBytes = kPRows * 128;               // 64 keys of all rows
    static constexpr int kPBytes = 2 * kPHalfBytes;
    static constexpr int kQHalfBytes = 2 * kCap * 128;             // 64 elements of D of two blocks' rows
    static constexpr int kQBytes = kHalves * kQHalfBytes;
    static constexpr int kCtlBytes = 512 + 10 * kCap * 4;          // barriers; two segments' references and sums
    static constexpr int kRoom = 232448 - kCtlBytes - 2 * kPBytes - kQBytes;
    static constexpr int kFit = kRoom / kTensorBytes;
    static constexpr int kSlotsK = (kFit + 1) / 2 < kMaxSlots ? (kFit + 1) / 2 : kMaxSlots;
    static constexpr int kSlotsV = kFit / 2 < kMaxSlots ? kFit / 2 : kMaxSlots;
    static constexpr int kVOff = kSlotsK * kTensorBytes;
    static constexpr int kPOff = kVOff + kSlotsV * kTensorBytes;   // (V's last tile is followed by P: see the products)
    static constexpr int kQOff = kPOff + 2 * kPBytes;
    static constexpr int kCtlOff = kQOff + kQBytes;
    static constexpr size_t kSmemBytes = kCtlOff + kCtlBytes;
    static constexpr int kOCol = 2 * kCap;                         // O twice, kPRows columns each, behind S twice
    static constexpr uint32_t kTmemCols = 8 * kCap;                // (a power of two)
};

struct Ctl {
    uint64_t k_full[kMaxSlots], k_empty[kMaxSlots], v_full[kMaxSlots], v_empty[kMaxSlots];
    uint64_t q_full[2], q_empty[2];
    uint64_t s_full[2];   // tensor core -> softmax: scores of a tile
    uint64_t p_ready[2];  // softmax -> tensor core: P is there, and the scores have been read
    uint64_t pv_done[2];  // a tile's product with V has been added (and its P read)
    uint64_t o_done[2];   // ... the last one of a segment
    uint64_t ml_ready[2]; // softmax -> output: the segment's maxima and sums are there
    uint64_t o_free[2];   // output -> tensor core and softmax: output, maxima and sums have been read
    uint64_t drain[2];
    uint32_t tmem_base, abort_flag, drain_flag, data_error;
};
static_assert(sizeof(Ctl) <= 512, "room of the barriers");

// Key tiles lie as [group of 8 keys][half][8 rows][128 bytes], swizzled: a 16-token page is one TMA box.
template <int D>
__device__ __forceinline__ uint32_t key_off(int r, int c) {  // of 16-byte chunk c of key r
    return static_cast<uint32_t>(((r >> 3) * (D / 64) + (c >> 3)) * 1024 + (r & 7) * 128 + (((c & 7) ^ (r & 7)) << 4));
}

__device__ __forceinline__ void team_sync(int id) { asm volatile("bar.sync %0, 128;" ::"r"(id) : "memory"); }
__device__ __forceinline__ bool team_any(int id, bool x) {
    uint32_t r;
    asm volatile(
        "{\n"
        " .reg .pred p, q;\n"
        " setp.ne.u32 p, %2, 0;\n"
        " bar.red.or.pred q, %1, 128, p;\n"
        " selp.u32 %0, 1, 0, q;\n"
        "}\n"
        : "=r"(r) : "r"(id), "r"(x ? 1u : 0u) : "memory");
    return r != 0u;
}

struct Maps {  // Q (boxes of one token, of as many as a block holds), K, V
    CUtensorMap q1, qb, k, v;
};

// One CTA's piece of the line.
template <int D, int kCap>
__global__ void __launch_bounds__(Layout<D, kCap>::kThreads, 1) group_tile_kernel(const __grid_constant__ Maps maps, const __grid_constant__ Params p) {
    using L = Layout<D, kCap>;
    constexpr int kTeams = L::kTeams, kProducerWarp = L::kProducerWarp, kScoreWarp = L::kScoreWarp, kValueWarp = L::kValueWarp, kQWarp = L::kQWarp, kOutWarp = L::kOutWarp;
    // 512 * 88 + 256 * 64 = 768 * 80, what a launch of 768 threads has
    constexpr int kSoftmaxRegs = L::kThreads == 768 ? 88 : 0, kOtherRegs = 64;
    extern __shared__ __align__(1024) uint8_t smem[];
    if ((smem_u32(smem) & 1023u) != 0u) {  // swizzled tiles need 1024-byte alignment; never expected
        if (threadIdx.x == 0 && p.status != nullptr) atomicCAS(p.status, 0, RPX_ERR_CUDA);
        return;
    }
    Ctl* ctl = reinterpret_cast<Ctl*>(smem + L::kCtlOff);
    // [O buffer][4 quarters' sums, reference][row] of a segment
    float* ml = reinterpret_cast<float*>(smem + L::kCtlOff + 512);
    volatile uint32_t* abort_flag = &ctl->abort_flag;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (threadIdx.x == 0) {
        for (int i = 0; i < kMaxSlots; ++i) {
            mbar_init(&ctl->k_full[i], 1);
            mbar_init(&ctl->k_empty[i], 1);
            mbar_init(&ctl->v_full[i], 1);
            mbar_init(&ctl->v_empty[i], 1);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(&ctl->q_full[i], 1);
            mbar_init(&ctl->q_empty[i], 1);
            mbar_init(&ctl->s_full[i], 1);
            mbar_init(&ctl->p_ready[i], 4 * kTeams);
            mbar_init(&ctl->pv_done[i], 1);
            mbar_init(&ctl->drain[i], 1);
            mbar_init(&ctl->o_done[i], 1);
            mbar_init(&ctl->ml_ready[i], 4 * kTeams);
            mbar_init(&ctl->o_free[i], 4);
        }
        ctl->abort_flag = ctl->drain_flag = ctl->data_error = 0;
        fence_barrier_init();
    }
    if (warp == kValueWarp) {
        tmem_alloc(&ctl->tmem_base, L::kTmemCols);
        tmem_relinquish();
    }
    tc_fence_before_sync();
    __syncthreads();
    tc_fence_after_sync();
    const uint32_t tmem_base = ctl->tmem_base;  // S at columns 0 and kCap, O at kOCol
    asm volatile("griddepcontrol.wait;" ::: "memory");  // the plan
    auto rows16 = [&](const auto& w) { return (w.tokens() * p.group + 15) & ~15; };

    if (warp == kProducerWarp) {
        // =========================================================== producer: K a tile ahead of V, through all segments
        if constexpr (kSoftmaxRegs > 0) asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kOtherRegs));
        Walk walk;
        walk.start(p, blockIdx.x);
        bool ok = true;
        uint32_t nk = 0, nv = 0;
        // the tile whose V comes next: page number of this lane's page, boxes, KV head
        int32_t v_block = 0, v_boxes = 0, v_head = 0;
        const int pg = lane & 7;
        auto load = [&](const CUtensorMap* map, uint8_t* dst, uint64_t* full, int32_t block, int32_t boxes, int32_t head) {
            if (lane == 0) mbar_arrive_expect_tx(full, static_cast<uint32_t>(boxes) * kPage * D * 2);
            __syncwarp();  // the byte count is armed before any copy can complete
            if (lane < boxes) tma_load_4d(dst + pg * (kPage * D * 2), map, full, 0, 0, 0, (block * p.num_kv_heads + head) * 2);
            __syncwarp();
        };
        auto load_v = [&]() {
            const uint32_t st = nv % L::kSlotsV;
            if (!mbar_wait(&ctl->v_empty[st], ((nv / L::kSlotsV) & 1u) ^ 1u, abort_flag)) return false;
            load(&maps.v, smem + L::kVOff + st * L::kTensorBytes, &ctl->v_full[st], v_block, v_boxes, v_head);
            ++nv;
            return true;
        };
        while (ok && walk.next(p)) {
            const int32_t* table = p.block_table + static_cast<int64_t>(walk.q.row) * p.block_table_stride + walk.q.page0;
            const int32_t pages = (walk.q.len - 1) / kPage + 1;  // (len + 15 may not fit 32 bits)
            auto read_block = [&](int32_t t) { return t < walk.t1 && t * kPages + pg < pages ? __ldg(table + t * kPages + pg) : 0; };
            int32_t next_block = read_block(walk.t0);
            for (int32_t t = walk.t0; t < walk.t1; ++t) {
                int32_t block = next_block;
                next_block = read_block(t + 1);
                if (block < 0 || block >= p.num_blocks) {
                    ctl->data_error = 1;
                    block = 0;
                }
                const int32_t boxes = min(kPages, pages - t * kPages);
                const uint32_t st = nk % L::kSlotsK;
                ok = mbar_wait(&ctl->k_empty[st], ((nk / L::kSlotsK) & 1u) ^ 1u, abort_flag);
                if (!ok) break;
                load(&maps.k, smem + st * L::kTensorBytes, &ctl->k_full[st], block, boxes, walk.head);
                ++nk;
                if (nk > 1) ok = load_v();
                if (!ok) break;
                v_block = block;
                v_boxes = boxes;
                v_head = walk.head;
            }
        }
        if (ok && nk > 0) ok = load_v();
        if (!ok) {  // abort: copies still in flight get a moment to land before shared memory is released
            for (uint32_t i = nk > L::kSlotsK ? nk - L::kSlotsK : 0u; i < nk; ++i)
                mbar_wait(&ctl->k_full[i % L::kSlotsK], (i / L::kSlotsK) & 1u, &ctl->drain_flag, kDrainLimitCycles);
            for (uint32_t i = nv > L::kSlotsV ? nv - L::kSlotsV : 0u; i < nv; ++i)
                mbar_wait(&ctl->v_full[i % L::kSlotsV], (i / L::kSlotsV) & 1u, &ctl->drain_flag, kDrainLimitCycles);
        }
    } else if (warp == kScoreWarp) {
        // =========================================================== S^T = K Q^T, by one thread
        if constexpr (kSoftmaxRegs > 0) asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kOtherRegs));
        Walk walk;
        walk.start(p, blockIdx.x);
        if (elect_one()) {
            const uint64_t k_desc = make_smem_desc_sw128(smem_u32(smem), 16, L::kHalves * 1024);
            const uint64_t q_desc = make_smem_desc_sw128(smem_u32(smem + L::kQOff), 16, 1024);
            bool ok = true;
            uint32_t segments = 0, tiles = 0;
            for (; ok && walk.next(p); ++segments) {
                const uint32_t qb = segments & 1u, idesc = make_idesc_bf16(128, rows16(walk), false, false);
                const uint64_t qd = q_desc + static_cast<uint64_t>(qb * kCap * 8);
                ok = mbar_wait(&ctl->q_full[qb], (segments >> 1) & 1u, abort_flag);
                for (int32_t t = walk.t0; ok && t < walk.t1; ++t, ++tiles) {
                    const uint32_t st = tiles % L::kSlotsK, b = tiles & 1u;
                    ok = (tiles < 2 || mbar_wait(&ctl->p_ready[b], ((tiles >> 1) - 1) & 1u, abort_flag)) &&
                         mbar_wait(&ctl->k_full[st], (tiles / L::kSlotsK) & 1u, abort_flag);
                    if (!ok) break;
                    tc_fence_after_sync();
                    const uint64_t kd = k_desc + static_cast<uint64_t>(st * (L::kTensorBytes >> 4));
#pragma unroll
                    for (int ks = 0; ks < D / 16; ++ks)
                        umma_bf16_ss(tmem_base + b * kCap, kd + (ks >> 2) * 64 + 2 * (ks & 3), qd + (ks >> 2) * (L::kQHalfBytes >> 4) + 2 * (ks & 3), idesc, ks != 0);
                    umma_commit(&ctl->s_full[b]);
                    umma_commit(&ctl->k_empty[st]);
                    if (t + 1 == walk.t1) umma_commit(&ctl->q_empty[qb]);
                }
            }
            if (!ok) {
                umma_commit(&ctl->drain[0]);
                mbar_wait(&ctl->drain[0], 0, &ctl->drain_flag, kDrainLimitCycles);
            }
        }
    } else if (warp == kValueWarp) {
        // =========================================================== O^T += V^T P^T, by one thread
        if constexpr (kSoftmaxRegs > 0) asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kOtherRegs));
        Walk walk;
        walk.start(p, blockIdx.x);
        if (elect_one()) {
            // D = 64: M stays 128, and the lanes 64 .. 127 of O^T, which nobody reads, are fed by whatever lies 1 KB on
            const uint64_t v_desc = make_smem_desc_sw128(smem_u32(smem + L::kVOff), 1024, L::kHalves * 1024);
            const uint64_t p_desc = make_smem_desc_sw128(smem_u32(smem + L::kPOff), 16, 1024);
            bool ok = true;
            uint32_t segments = 0, tiles = 0;
            while (ok && walk.next(p)) {
                const uint32_t ob = segments & 1u, idesc = make_idesc_bf16(128, 2 * rows16(walk), true, false);
                if (segments >= 2) ok = mbar_wait(&ctl->o_free[ob], ((segments >> 1) - 1) & 1u, abort_flag);
                for (int32_t t = walk.t0; ok && t < walk.t1; ++t, ++tiles) {
                    const uint32_t b = tiles & 1u, st = tiles % L::kSlotsV;
                    ok = mbar_wait(&ctl->v_full[st], (tiles / L::kSlotsV) & 1u, abort_flag) && mbar_wait(&ctl->p_ready[b], (tiles >> 1) & 1u, abort_flag);
                    if (!ok) break;
                    tc_fence_after_sync();
                    const int32_t steps = (min(kTile, walk.q.len - t * kTile) + 15) / 16;  // pages that were loaded
                    const uint64_t vd = v_desc + static_cast<uint64_t>(st * (L::kTensorBytes >> 4)), pd = p_desc + static_cast<uint64_t>(b * (L::kPBytes >> 4));
#pragma unroll
                    for (int32_t ks = 0; ks < kTile / 16; ++ks)
                        if (ks < steps)
                            umma_bf16_ss(tmem_base + L::kOCol + ob * L::kPRows, vd + static_cast<uint64_t>(ks * (L::kHalves * 128)),
                                         pd + static_cast<uint64_t>((ks >> 2) * (L::kPHalfBytes >> 4) + 2 * (ks & 3)), idesc, t != walk.t0 || ks != 0);
                    umma_commit(&ctl->v_empty[st]);
                    umma_commit(&ctl->pv_done[b]);
                    if (t + 1 == walk.t1) umma_commit(&ctl->o_done[ob]);
                }
                ++segments;
            }
            if (!ok) {
                umma_commit(&ctl->drain[1]);
                mbar_wait(&ctl->drain[1], 0, &ctl->drain_flag, kDrainLimitCycles);
            }
        }
        __syncwarp();
        // the join may start on the SMs that become free
        asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    } else if (warp == kQWarp) {
        // =========================================================== Q of a segment's block
        // One box lands as consecutive 128-byte rows: of one token, or of as many as a block holds.
        // (What lies behind the block's rows is another token's, or was there before: those rows are nobody's.)
        if constexpr (kSoftmaxRegs > 0) asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kOtherRegs));
        Walk walk;
        walk.start(p, blockIdx.x);
        if (elect_one()) {
            uint32_t segments = 0;
            bool ok = true;
            for (; walk.next(p); ++segments) {
                const uint32_t qb = segments & 1u;
                ok = segments < 2 || mbar_wait(&ctl->q_empty[qb], ((segments >> 1) - 1) & 1u, abort_flag);
                if (!ok) break;
                const bool one = walk.tokens() == 1;
                mbar_arrive_expect_tx(&ctl->q_full[qb], static_cast<uint32_t>((one ? 1 : kCap / p.group) * p.group * L::kHalves) * 128);
                for (int hf = 0; hf < L::kHalves; ++hf)
                    tma_load_3d(smem + L::kQOff + hf * L::kQHalfBytes + qb * kCap * 128, one ? &maps.q1 : &maps.qb, &ctl->q_full[qb], hf * 64, walk.head * p.step,
                                walk.q.tok0 + walk.token0());
            }
            if (!ok)  // abort: the copies in flight get a moment to land
                for (uint32_t i = segments > 2 ? segments - 2 : 0u; i < segments; ++i)
                    mbar_wait(&ctl->q_full[i & 1u], (i >> 1) & 1u, &ctl->drain_flag, kDrainLimitCycles);
        }
    } else if (warp >= kOutWarp && warp < kOutWarp + 4) {
        // =========================================================== output: a warp 32 elements of D of all rows
        if constexpr (kSoftmaxRegs > 0) asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kOtherRegs));
        Walk walk;
        walk.start(p, blockIdx.x);
        const int quarter = warp & 3;
        const int32_t d = quarter * 32 + lane;
        uint32_t segments = 0;
        bool ok = true;
        while (walk.next(p)) {
            const uint32_t ob = segments & 1u;
            const int32_t rows = walk.tokens() * p.group;
            const bool own = walk.e >= p.n_groups, whole = walk.t0 == 0 && walk.t1 == walk.q.tiles;
            const bool last_word = whole && own && walk.q.page0 == 0;  // nothing to add: this is the result
            // where the block's rows go: in order in a slot, or each in its own place
            const int64_t first_row = (static_cast<int64_t>(walk.q.tok0) + walk.token0()) * p.num_q_heads + walk.head * p.step;
            const int64_t base = whole ? (own && !last_word ? p.total_tokens * p.num_q_heads : 0) + first_row : (static_cast<int64_t>(blockIdx.x) * 2 + (walk.t0 == 0 ? 1 : 0)) * kCap;
            const int32_t skip = whole ? p.num_q_heads - p.group : 0;  // rows between a token's last and the next one's first
            float* dst = (whole ? p.whole_o : p.part_o) + base * D + d;
            __nv_bfloat16* out = static_cast<__nv_bfloat16*>(p.out) + base * D + d;
            float2* dst_ml = (whole ? p.whole_ml : p.part_ml) + base;
            const float* now = ml + ob * 5 * kCap + lane;
            const int32_t n16 = rows16(walk);
            const uint32_t o_addr = tmem_base + L::kOCol + ob * L::kPRows + (static_cast<uint32_t>(quarter * 32) << 16);
            if (!mbar_wait(&ctl->ml_ready[ob], (segments >> 1) & 1u, abort_flag)) break;
            for (int32_t r0 = 0; r0 < rows; r0 += 32, now += 32) {  // 32 rows a turn, a lane's numbers are those of row r0 + lane
                const int32_t here = min(32, rows - r0);
                int32_t at = 0;
                float inv = 0.f;
                if (lane < here) {
                    const float total = (now[0] + now[kCap]) + (now[2 * kCap] + now[3 * kCap]), m = now[4 * kCap];
                    at = r0 + lane + over_group(p, r0 + lane) * skip;
                    inv = 1.f / total;
                    if (quarter == 0) {
                        if (!last_word) dst_ml[at] = make_float2(m, total);
                        else if (p.lse != nullptr) p.lse[base + at] = (m + log2f(total)) * kLn2;
                    }
                }
                if (r0 == 0) {
                    if (!mbar_wait(&ctl->o_done[ob], (segments >> 1) & 1u, abort_flag)) {
                        ok = false;
                        break;
                    }
                    tc_fence_after_sync();
                }
                if (d >= D) continue;
                int32_t place = r0 + over_group(p, r0) * skip, in_group = r0 - over_group(p, r0) * p.group;  // of the next row
#pragma unroll 1
                for (int32_t c = 0; c < here; c += 8) {
                    uint32_t o[8], lo[8];
                    tmem_ld8(o_addr + r0 + c, o);
                    tmem_ld8(o_addr + n16 + r0 + c, lo);
                    tmem_ld_wait();
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const float x = __uint_as_float(o[i]) + __uint_as_float(lo[i]);
                        const float f = last_word ? __shfl_sync(0xffffffffu, inv, c + i) : 1.f;
                        if (c + i < here) {
                            if (last_word) out[static_cast<int64_t>(place) * D] = __float2bfloat16_rn(x * f);
                            else dst[static_cast<int64_t>(place) * D] = x;
                        }
                        ++place;
                        if (++in_group == p.group) {
                            in_group = 0;
                            place += skip;
                        }
                    }
                }
            }
            if (!ok) break;
            tc_fence_before_sync();
            __syncwarp();
            if (lane == 0) mbar_arrive(&ctl->o_free[ob]);
            ++segments;
        }
    } else if (warp < kProducerWarp) {
        // =========================================================== softmax
        // After a wait that ran out (ok == false) a warp goes through the rest of its walk without waiting: every warp still meets
        // the others at the same barriers, and the outputs of the call are undefined anyway.
        if constexpr (kSoftmaxRegs > 0) asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kSoftmaxRegs));
        Walk walk;
        walk.start(p, blockIdx.x);
        constexpr int kBlocks = L::kBlocks;
        const int team = warp >> 2, quarter = warp & 3, bar = 1 + team;
        const uint32_t lane_addr = static_cast<uint32_t>(quarter * 32) << 16;
        const int key0 = quarter * 32 + (lane >> 2);            // this thread's keys of a tile: key0 + 8 m
        const int pair = 2 * (lane & 3);                        // its rows of an 8-row block: pair, pair + 1
        uint32_t tiles = 0, segments = 0;
        int32_t turn = 0;
        bool ok = true;
        while (walk.next(p)) {
            const int32_t len = walk.q.len, tokens = walk.tokens(), token0 = walk.token0(), rows = tokens * p.group, n16 = (rows + 15) & ~15;
            // the block's rows by eights, kBlocks of these to a team; a segment begins with the team behind the last one's, so that
            // small segments go to the teams in turn.  (Nobody writes P's rows beyond: their outputs are nobody's.)
            const int32_t eights = (rows + 7) / 8, mine = (team - turn) & (kTeams - 1);
            const int32_t nb = min(kBlocks, eights - mine * kBlocks), row0 = 8 * mine * kBlocks;
            turn += (eights + kBlocks - 1) / kBlocks;
            const bool own = walk.e >= p.n_groups;
            const int32_t seen_by_first = own ? len - walk.q.n + token0 + 1 : len;  // keys that the block's first token sees
            // of the pairs of rows that this thread holds: what a score has to pass for the reference to be raised (rows that are
            // nobody's never do), the reference with its sign turned (0 for a row that has seen no key), and the sum over the
            // thread's keys
            float limit[2 * kBlocks], base[2 * kBlocks], sum[2 * kBlocks];
#pragma unroll
            for (int i = 0; i < 2 * kBlocks; ++i) {
                limit[i] = row0 + 8 * (i >> 1) + pair + (i & 1) < rows ? -CUDART_INF_F : CUDART_INF_F;
                base[i] = sum[i] = 0.f;
            }
            auto reference = [&](int i) { return limit[i] == -CUDART_INF_F ? -CUDART_INF_F : -base[i]; };
            // (All kBlocks are gone through whether they have rows or not: a form for every number of them is more code than the
            // instruction cache holds beside the other roles', and took twice as long.)
            for (int32_t t = walk.t0; t < walk.t1; ++t, ++tiles) {
                const uint32_t b = tiles & 1u;
                const bool first = t == walk.t0;
                if (ok) ok = mbar_wait(&ctl->s_full[b], (tiles >> 1) & 1u, abort_flag);
                tc_fence_after_sync();
                const int32_t left = len - t * kTile;  // keys from the tile's first on
                if (nb > 0) {
                uint32_t sc[kBlocks][8];  // [block][2 m + row of the pair]: key m
#pragma unroll
                for (int k = 0; k < kBlocks; ++k) {
                    tmem_ld_16x256(tmem_base + b * kCap + row0 + 8 * k + lane_addr, &sc[k][0]);
                    tmem_ld_16x256(tmem_base + b * kCap + row0 + 8 * k + lane_addr + (16u << 16), &sc[k][4]);
                }
                tmem_ld_wait();
                if (left < kTile || seen_by_first - t * kTile < kTile) {
#pragma unroll
                    for (int k = 0; k < kBlocks; ++k)
#pragma unroll
                        for (int e = 0; e < 2; ++e) {
                            const int32_t token = min(over_group(p, row0 + 8 * k + pair + e), tokens - 1);
                            const int32_t seen = min(left, seen_by_first - t * kTile + token);  // (in this order: the sum of the first two may not fit)
#pragma unroll
                            for (int m = 0; m < 4; ++m)
                                if (key0 + 8 * m >= seen) sc[k][2 * m + e] = 0xff800000u;  // -inf
                        }
                }
                // its P has been read: until P is written, its place is where the team's warps exchange numbers, [5][rows]
                if (ok && tiles >= 2) ok = mbar_wait(&ctl->pv_done[b], ((tiles >> 1) - 1) & 1u, abort_flag);
                float* all = reinterpret_cast<float*>(smem + L::kPOff + b * L::kPBytes + row0 * 128);
                auto top_of = [&](int k, int e) {
                    return fmaxf(fmax3(__uint_as_float(sc[k][e]), __uint_as_float(sc[k][2 + e]), __uint_as_float(sc[k][4 + e])), __uint_as_float(sc[k][6 + e]));
                };
                // ---- does any row's reference have to be raised?
                bool up = first;
#pragma unroll
                for (int k = 0; k < kBlocks; ++k)
#pragma unroll
                    for (int e = 0; e < 2; ++e) up |= top_of(k, e) > limit[2 * k + e];
                if (team_any(bar, up)) {
#pragma unroll
                    for (int k = 0; k < kBlocks; ++k)
#pragma unroll
                        for (int e = 0; e < 2; ++e) {
                            float top = top_of(k, e);
#pragma unroll
                            for (int off = 4; off < 32; off <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, off));
                            if (lane < 4) all[(quarter * kBlocks + k) * 8 + pair + e] = top;
                        }
                    team_sync(bar);
                    float keep[2 * kBlocks];
#pragma unroll
                    for (int k = 0; k < kBlocks; ++k)
#pragma unroll
                        for (int e = 0; e < 2; ++e) {
                            const int r = 8 * k + pair + e;
                            const float top = fmaxf(fmaxf(all[r], all[8 * kBlocks + r]), fmaxf(all[16 * kBlocks + r], all[24 * kBlocks + r])) * p.scale_log2;
                            const float old = reference(2 * k + e);
                            const bool raise = top > old + kRaise;
                            const float now = raise ? top : old;
                            keep[2 * k + e] = raise ? fast_exp2(old - top) : 1.f;  // (from -inf: 0)
                            sum[2 * k + e] *= keep[2 * k + e];
                            base[2 * k + e] = now == -CUDART_INF_F ? 0.f : -now;
                            if (row0 + r < rows) limit[2 * k + e] = (now + kRaise) / p.scale_log2;
                        }
                    if (!first) {  // what O holds goes along
                        if (quarter == 0 && lane < 4) {
#pragma unroll
                            for (int k = 0; k < kBlocks; ++k)
#pragma unroll
                                for (int e = 0; e < 2; ++e) all[32 * kBlocks + 8 * k + pair + e] = keep[2 * k + e];
                        }
                        team_sync(bar);
                        if (ok) ok = mbar_wait(&ctl->pv_done[b ^ 1u], ((tiles - 1) >> 1) & 1u, abort_flag);
                        tc_fence_after_sync();
#pragma unroll 1
                        for (int c = 0; c < 8 * nb; c += 8) {
                            uint32_t o[8];
                            const uint32_t at = tmem_base + L::kOCol + (segments & 1u) * L::kPRows + row0 + c + lane_addr;
                            tmem_ld8(at, o);
                            tmem_ld_wait();
#pragma unroll
                            for (int i = 0; i < 8; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * all[32 * kBlocks + c + i]);
                            tmem_st8(at, o);
                            tmem_ld8(at + n16, o);
                            tmem_ld_wait();
#pragma unroll
                            for (int i = 0; i < 8; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * all[32 * kBlocks + c + i]);
                            tmem_st8(at + n16, o);
                        }
                        tmem_st_wait();
                    }
                    team_sync(bar);  // the exchange has been read
                }
                // ---- P = 2^(s - reference): 0 for a masked key (-inf), NaN for NaN and for +inf (inf - inf)
                const uint32_t pb = smem_u32(smem + L::kPOff + b * L::kPBytes + (quarter >> 1) * L::kPHalfBytes);
                const int chunk = (quarter & 1) * 4 + (lane >> 3), prow = row0 + (lane & 7);
                const uint32_t at0 = pb + prow * 128 + ((chunk ^ (prow & 7)) << 4);  // (row0 is a multiple of 8)
                const uint64_t scale2 = f2_pack(p.scale_log2, p.scale_log2);
#pragma unroll
                for (int k = 0; k < kBlocks; ++k) {
                    const uint64_t base2 = f2_pack(base[2 * k], base[2 * k + 1]);
                    uint32_t hi[4];
                    uint64_t x[4];
#pragma unroll
                    for (int m = 0; m < 4; ++m) {
                        float x0, x1;
                        f2_unpack(f2_fma(f2_pack(__uint_as_float(sc[k][2 * m]), __uint_as_float(sc[k][2 * m + 1])), scale2, base2), x0, x1);
                        x0 = fast_exp2(x0);
                        x1 = fast_exp2(x1);
                        x[m] = f2_pack(x0, x1);
                        hi[m] = pack_bf16x2(x0, x1);
                        sc[k][2 * m] = __float_as_uint(x0);
                        sc[k][2 * m + 1] = __float_as_uint(x1);
                    }
                    f2_unpack(f2_add(f2_pack(sum[2 * k], sum[2 * k + 1]), f2_add(f2_add(x[0], x[1]), f2_add(x[2], x[3]))), sum[2 * k], sum[2 * k + 1]);
                    if (kBlocks == 1 || k < nb) stsm_x4_trans(at0 + 8 * k * 128, hi[0], hi[1], hi[2], hi[3]);
                }
#pragma unroll
                for (int k = 0; k < kBlocks; ++k) {  // what that rounding dropped
                    uint32_t lo[4];
#pragma unroll
                    for (int m = 0; m < 4; ++m) {
                        const float x0 = __uint_as_float(sc[k][2 * m]), x1 = __uint_as_float(sc[k][2 * m + 1]);
                        const uint32_t hi = pack_bf16x2(x0, x1);
                        lo[m] = pack_bf16x2(x0 - __uint_as_float(hi << 16), x1 - __uint_as_float(hi & 0xffff0000u));
                    }
                    if (kBlocks == 1 || k < nb) stsm_x4_trans(at0 + (8 * k + n16) * 128, lo[0], lo[1], lo[2], lo[3]);
                }
                }
                // ---- V's rows behind the last key of a page that was loaded may hold anything: a probability of 0 must not
                // meet a NaN there
                const int32_t ragged = left < kTile ? left & 15 : 0;
                if (ragged != 0) {
                    const uint32_t st = tiles % L::kSlotsV;
                    // (The product two tiles before has been waited for by teams with rows; without that wait the slot may still be an
                    // earlier tile's, and the barrier's parity cannot tell the two.)
                    if (ok && tiles >= 2) ok = mbar_wait(&ctl->pv_done[b], ((tiles >> 1) - 1) & 1u, abort_flag);
                    if (ok) ok = mbar_wait(&ctl->v_full[st], (tiles / L::kSlotsV) & 1u, abort_flag);
                    uint8_t* v = smem + L::kVOff + st * L::kTensorBytes;
                    for (int32_t i = threadIdx.x; i < (16 - ragged) * (D / 8); i += 128 * kTeams)
                        *reinterpret_cast<uint4*>(v + key_off<D>(left + i / (D / 8), i % (D / 8))) = make_uint4(0u, 0u, 0u, 0u);
                }
                fence_proxy_async_smem();
                tc_fence_before_sync();
                __syncwarp();
                if (lane == 0) mbar_arrive(&ctl->p_ready[b]);
            }
            // ---- the segment's references and this warp's sums, for the output warps
            const uint32_t ob = segments & 1u;
            if (ok && segments >= 2) ok = mbar_wait(&ctl->o_free[ob], ((segments >> 1) - 1) & 1u, abort_flag);
            float* to = ml + (ob * 5 + quarter) * kCap + row0;
#pragma unroll
            for (int k = 0; k < kBlocks; ++k)
                if (k < nb) {
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        float x = sum[2 * k + e];
#pragma unroll
                        for (int off = 4; off < 32; off <<= 1) x += __shfl_xor_sync(0xffffffffu, x, off);
                        if (lane < 4) to[8 * k + pair + e] = x;
                        if (quarter == 0 && lane < 4) to[4 * kCap + 8 * k + pair + e] = reference(2 * k + e);
                    }
                }
            __syncwarp();
            if (lane == 0) mbar_arrive(&ctl->ml_ready[ob]);
            ++segments;
        }
    }
    tc_fence_before_sync();
    __syncthreads();
    if (warp == kValueWarp) {
        tc_fence_after_sync();
        tmem_dealloc(tmem_base, L::kTmemCols);
    }
    if (threadIdx.x == 0 && p.status != nullptr) {
        if (ctl->abort_flag != 0u) atomicCAS(p.status, 0, RPX_ERR_TIMEOUT);
        else if (ctl->data_error != 0u) atomicCAS(p.status, 0, RPX_ERR_DEVICE_DATA);
    }
}

template <int D, int kCap>
rpx_status_t make_maps(Maps* m, const Params& p, const rpx_kv_cache_t& cache) {
    using L = Layout<D, kCap>;
    static_assert(L::kSlotsK >= 2 && L::kSlotsV >= 2 && L::kSmemBytes <= 232448, "shared memory of one CTA");
    static_assert(L::kTmemCols >= 32 && L::kTmemCols <= 512, "tensor memory");
    {
        // a block's rows as (64 elements, heads of a KV head, tokens); a part's last KV head has p.group heads left
        const uint64_t dims[3] = {D, static_cast<uint64_t>((p.num_kv_heads - 1) * p.step + p.group), static_cast<uint64_t>(p.total_tokens)};
        const uint64_t strides[2] = {D * 2ull, static_cast<uint64_t>(p.q_stride) * 2};
        uint32_t box[3] = {64, static_cast<uint32_t>(p.group), 1};
        if (rpx_status_t rc = encode_tmap_bf16(&m->q1, p.q, 3, dims, strides, box)) return rc;
        box[2] = static_cast<uint32_t>(kCap / p.group);
        if (rpx_status_t rc = encode_tmap_bf16(&m->qb, p.q, 3, dims, strides, box)) return rc;
    }
    // the pool as groups of 8 keys: two per page and head
    const uint64_t groups = static_cast<uint64_t>(cache.num_blocks) * p.num_kv_heads * 2;  // (fits 32 bits: checked by the caller)
    const uint64_t dims[4] = {64, 8, D / 64, groups};
    const uint64_t strides[3] = {D * 2ull, 128, 8 * D * 2ull};
    const uint32_t box[4] = {64, 8, D / 64, 2};
    if (rpx_status_t rc = encode_tmap_bf16(&m->k, cache.k_cache, 4, dims, strides, box)) return rc;
    return encode_tmap_bf16(&m->v, cache.v_cache, 4, dims, strides, box);
}

template <int D, int kCap>
rpx_status_t launch_one(const Params& p, const rpx_kv_cache_t& cache, cudaStream_t stream) {
    using L = Layout<D, kCap>;
    Maps maps;
    if (rpx_status_t rc = make_maps<D, kCap>(&maps, p, cache)) return rc;
    auto* kernel = group_tile_kernel<D, kCap>;
    if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(L::kSmemBytes)) != cudaSuccess) return RPX_ERR_CUDA;
    return launch_on_top(kernel, static_cast<unsigned>(p.ctas), L::kThreads, L::kSmemBytes, stream, maps, p);
}
template <int D>
rpx_status_t launch_cap(const Params& p, const rpx_kv_cache_t& cache, cudaStream_t stream) {
    switch (p.cap) {
        case 16: return launch_one<D, 16>(p, cache, stream);
        case 32: return launch_one<D, 32>(p, cache, stream);
        default: return launch_one<D, kMostRows>(p, cache, stream);
    }
}

}  // namespace

namespace group {
rpx_status_t launch_group_tile(const Params& p, int32_t head_dim, const rpx_kv_cache_t& cache, cudaStream_t stream) {
    return head_dim == 128 ? launch_cap<128>(p, cache, stream) : launch_cap<64>(p, cache, stream);
}
}  // namespace group

}  // namespace rpx
