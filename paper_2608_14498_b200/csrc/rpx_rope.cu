// Per-head RMS norm of queries and keys with the rotation by multi-axis positions in the same pass, and its backward.
//
//   u = x * r,  r = (mean(x^2) + eps)^(-1/2),  y = u * w     (both steps left out when the weights are NULL)
//   pair i = (i, i + rot/2) of the first rot elements is turned by theta_i = position[axis(i)] * inv_freq[i]:
//   out_i = y_i cos - y_{i+rot/2} sin,  out_{i+rot/2} = y_{i+rot/2} cos + y_i sin;  the elements from rot on pass through
//
// backward, with g = (transposed rotation) dout:
//   dw = sum over tokens and heads of g * u,   dx = r * (g w - u * mean(g w u))
//
// Bound by memory: 2 + 2 bytes per value forward in bf16, 2 + 4 + 2 backward (the gradients that arrive are float32).
// A row of head_dim values is held by head_dim / 16 lanes, each with TWO 8-element chunks: the two that the rotation
// pairs up (p and p + rot/16; beyond rot two neighbours), so neither half ever moves between lanes and the only
// exchange is the sum of squares.  A warp keeps one token: its rot/2 angles are computed once, two per lane, and read
// back from shared memory as the lane's eight (cos, sin) pairs for all of the token's heads.
//
// Measured with 28 + 4 heads of 128, bf16, inputs beyond L2: forward of 32768 tokens 86 us, backward of 34816 tokens 183 us,
// both 95 % of the copy bandwidth.  float32: forward of 8192 tokens 48 us (86 %), of 32768 172 us (95 %); backward 79 us
// (78 %) and 270 us (91 %).
#include <cuda_bf16.h>

#include "rpx_internal.h"
#include "rpx_ptx.cuh"

namespace rpx {

namespace {

constexpr int kWarps = 4;
constexpr int kMaxPairs = 64;

struct Params {
    const void *q, *k;
    void *q_out, *k_out;
    int64_t q_stride, k_stride, q_out_stride, k_out_stride;  // elements between tokens
    const void *q_weight, *k_weight;  // [D], or NULL
    const int32_t* positions;         // [axes][pos_stride]
    int64_t pos_stride;
    const float* inv_freq;            // [rot / 2]
    int64_t n_tokens;
    int32_t num_q_heads, num_kv_heads, rot;
    int32_t units_q, units, units_per_warp, warps_per_token;  // a unit = the rows one warp holds at once
    float eps;
    bool wide;                        // every float32 tensor starts on 32 bytes
    const float *dq, *dk;             // backward: [tokens][heads][D] contiguous
    float* dw_partial;                // backward: [grid][2][D], or NULL
    uint8_t axis[kMaxPairs];
};

// cos and sin of this token's angles.  The angle is reduced in 64 bits (position * frequency loses whole radians in 32
// bits at far positions): in units of half a turn, brought into [-1, 1], which 32 bits hold to 2^-25 of a half turn.
__device__ __forceinline__ void token_angles(const Params& p, int64_t token, int lane, float2* cs) {
    for (int i = lane; i < (p.rot >> 1); i += 32) {
        const double pos = static_cast<double>(__ldg(p.positions + p.axis[i] * p.pos_stride + token));
        const double half_turns = pos * (static_cast<double>(__ldg(p.inv_freq + i)) * 0.31830988618379067154);
        const float x = static_cast<float>(half_turns - 2.0 * rint(half_turns * 0.5));
        float s, c;
        sincospif(x, &s, &c);
        cs[((i & 7) >> 1) * (kMaxPairs / 4) + (i >> 3) * 2 + (i & 1)] = make_float2(c, s);
    }
    __syncwarp();
}

struct Bf16 {
    typedef __nv_bfloat16 Elem;
    typedef uint4 Raw;  // 8 elements
    static __device__ __forceinline__ Raw load(const Elem* p, bool) { return __ldcs(reinterpret_cast<const uint4*>(p)); }
    static __device__ __forceinline__ Raw zero() { return make_uint4(0u, 0u, 0u, 0u); }
    static __device__ __forceinline__ void unpack(const Raw& r, uint64_t (&x)[4]) {
        const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = f2_pack(__uint_as_float(w[i] << 16), __uint_as_float(w[i] & 0xffff0000u));
    }
    // the one rounding of the pass: results to bf16, nearest-even
    static __device__ __forceinline__ void store(Elem* p, const uint64_t (&x)[4], bool) {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float lo, hi;
            f2_unpack(x[i], lo, hi);
            w[i] = pack_bf16x2(lo, hi);
        }
        __stcs(reinterpret_cast<uint4*>(p), make_uint4(w[0], w[1], w[2], w[3]));
    }
};

// A lane's eight floats are one 32-byte access: as two of 16 bytes, every request of a warp would touch all of its sectors
// by halves, and the L1's request rate would bound the backward pass (it was 79 % busy when measured so, at 215 us for
// 34816 tokens of 28 + 4 heads of 128; see the top for what the pass takes now).
struct F32 {
    typedef float Elem;
    struct Raw { float v[8]; };
    static __device__ __forceinline__ Raw load(const Elem* p, bool wide) {
        Raw r;
        if (wide) {
            ld_global_v8(p, r.v);
        } else {
            const float4 a = reinterpret_cast<const float4*>(p)[0], b = reinterpret_cast<const float4*>(p)[1];
            r.v[0] = a.x; r.v[1] = a.y; r.v[2] = a.z; r.v[3] = a.w;
            r.v[4] = b.x; r.v[5] = b.y; r.v[6] = b.z; r.v[7] = b.w;
        }
        return r;
    }
    static __device__ __forceinline__ Raw zero() { return Raw{{0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f}}; }
    static __device__ __forceinline__ void unpack(const Raw& r, uint64_t (&x)[4]) {
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = f2_pack(r.v[2 * i], r.v[2 * i + 1]);
    }
    static __device__ __forceinline__ void store(Elem* p, const uint64_t (&packed)[4], bool wide) {
        float x[8];
#pragma unroll
        for (int i = 0; i < 4; ++i) f2_unpack(packed[i], x[2 * i], x[2 * i + 1]);
        if (wide) {
            st_global_v8(p, __float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3]),
                         __float_as_uint(x[4]), __float_as_uint(x[5]), __float_as_uint(x[6]), __float_as_uint(x[7]));
        } else {
            reinterpret_cast<float4*>(p)[0] = make_float4(x[0], x[1], x[2], x[3]);
            reinterpret_cast<float4*>(p)[1] = make_float4(x[4], x[5], x[6], x[7]);
        }
    }
};

// Sum over the lanes that hold one row.
template <int kLanes>
__device__ __forceinline__ float row_sum(float x) {
#pragma unroll
    for (int off = kLanes / 2; off > 0; off >>= 1) x += __shfl_xor_sync(0xffffffffu, x, off);
    return x;
}

// Where a lane's two chunks lie in a row.
template <int D>
struct LaneMap {
    static constexpr int kLanes = D / 16;      // lanes per row
    static constexpr int kRows = 32 / kLanes;  // rows (heads) a warp holds at once: one unit
    int row, off_a, off_b;
    bool turned;
    __device__ __forceinline__ LaneMap(int lane, int rot) {
        const int c = lane % kLanes, n = rot / 16;
        row = lane / kLanes;
        turned = c < n;
        off_a = 8 * (turned ? c : 2 * n + 2 * (c - n));
        off_b = turned ? off_a + rot / 2 : off_a + 8;
    }
};

// All arithmetic runs on packed pairs of floats, one instruction for two: the backward pass was short of issue slots
// (207 us with single floats, 183 with pairs).
__device__ __forceinline__ uint64_t f2_negate(uint64_t x) { return x ^ 0x8000000080000000ull; }
__device__ __forceinline__ float f2_sum(uint64_t x) {
    float lo, hi;
    f2_unpack(x, lo, hi);
    return lo + hi;
}

// A lane's eight cosines and sines, and a chunk of eight weights, out of shared memory.
__device__ __forceinline__ void read_angles(const float2* cs, int chunk, uint64_t (&c)[4], uint64_t (&s)[4]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float4 w = *reinterpret_cast<const float4*>(cs + i * (kMaxPairs / 4) + chunk * 2);
        c[i] = f2_pack(w.x, w.z);
        s[i] = f2_pack(w.y, w.w);
    }
}
template <int D>
__device__ __forceinline__ void read_weights(const float* w, int chunk, uint64_t (&x)[4]) {  // [half of a chunk][chunk][4]
    const float4 u = *reinterpret_cast<const float4*>(w + chunk * 4), v = *reinterpret_cast<const float4*>(w + D / 2 + chunk * 4);
    x[0] = f2_pack(u.x, u.y);
    x[1] = f2_pack(u.z, u.w);
    x[2] = f2_pack(v.x, v.y);
    x[3] = f2_pack(v.z, v.w);
}

// The weights as float32 in shared memory; called by the whole block, ends with a barrier.
template <class T, int D>
__device__ __forceinline__ void stage_weights(const Params& p, float (*w)[D]) {
    for (int i = threadIdx.x; i < 2 * D / 8; i += kWarps * 32) {
        uint64_t x[4];
        T::unpack(T::load(static_cast<const typename T::Elem*>(i < D / 8 ? p.q_weight : p.k_weight) + (i % (D / 8)) * 8, false), x);
#pragma unroll
        for (int e = 0; e < 4; ++e) *reinterpret_cast<uint64_t*>(&w[i / (D / 8)][(e >> 1) * (D / 2) + (i % (D / 8)) * 4 + 2 * (e & 1)]) = x[e];
    }
    __syncthreads();
}

// The loads run a batch ahead of the arithmetic, the first batch in front of the angles: a warp always has rows in flight.
template <class T, int D, bool kNorm>
__global__ void __launch_bounds__(kWarps * 32, sizeof(typename T::Elem) == 2 ? 6 : 4) qk_rope_kernel(const __grid_constant__ Params p) {
    typedef LaneMap<D> Map;
    typedef typename T::Elem Elem;
    constexpr int kUnroll = sizeof(Elem) == 2 ? 2 : 1;  // units of a batch
    __shared__ __align__(16) float2 cs_all[kWarps][kMaxPairs];
    __shared__ __align__(16) float weight[kNorm ? 2 : 1][D];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int64_t task = static_cast<int64_t>(blockIdx.x) * kWarps + warp;
    const int64_t token = task / p.warps_per_token;
    const int32_t u_begin = static_cast<int32_t>(task - token * p.warps_per_token) * p.units_per_warp;
    const int32_t u_end = token < p.n_tokens ? min(p.units, u_begin + p.units_per_warp) : 0;
    const Map map(lane, p.rot);
    const Elem* const q = static_cast<const Elem*>(p.q) + token * p.q_stride;
    const Elem* const k = static_cast<const Elem*>(p.k) + token * p.k_stride;

    typename T::Raw now[kUnroll][2], next[kUnroll][2];
    auto load = [&](typename T::Raw (&raw)[kUnroll][2], int32_t u0) {
#pragma unroll
        for (int i = 0; i < kUnroll; ++i) {
            const bool is_q = u0 + i < p.units_q;
            const int32_t head = (u0 + i - (is_q ? 0 : p.units_q)) * Map::kRows + map.row;
            const Elem* src = (is_q ? q : k) + head * D;
            const bool there = u0 + i < u_end && head < (is_q ? p.num_q_heads : p.num_kv_heads);
            raw[i][0] = there ? T::load(src + map.off_a, p.wide) : T::zero();
            raw[i][1] = there ? T::load(src + map.off_b, p.wide) : T::zero();
        }
    };
    load(now, u_begin);
    if (u_begin < u_end) token_angles(p, token, lane, cs_all[warp]);
    if (kNorm) stage_weights<T, D>(p, weight);
    if (u_begin >= u_end) return;
    uint64_t c[4], s[4];
    if (map.turned) read_angles(cs_all[warp], map.off_a >> 3, c, s);

    for (int32_t u0 = u_begin; u0 < u_end; u0 += kUnroll) {
        load(next, u0 + kUnroll);
#pragma unroll
        for (int i = 0; i < kUnroll; ++i) {
            if (u0 + i >= u_end) break;
            const bool is_q = u0 + i < p.units_q;
            const int32_t head = (u0 + i - (is_q ? 0 : p.units_q)) * Map::kRows + map.row;
            uint64_t a[4], b[4];
            T::unpack(now[i][0], a);
            T::unpack(now[i][1], b);
            if (kNorm) {
                uint64_t ss = 0ull, st = 0ull;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    ss = f2_fma(a[e], a[e], ss);
                    st = f2_fma(b[e], b[e], st);
                }
                const float r = rsqrtf(row_sum<Map::kLanes>(f2_sum(f2_add(ss, st))) * (1.f / D) + p.eps);
                const uint64_t r2 = f2_pack(r, r);
                uint64_t w[4];
                read_weights<D>(weight[is_q ? 0 : 1], map.off_a >> 3, w);
#pragma unroll
                for (int e = 0; e < 4; ++e) a[e] = f2_mul(f2_mul(a[e], r2), w[e]);
                read_weights<D>(weight[is_q ? 0 : 1], map.off_b >> 3, w);
#pragma unroll
                for (int e = 0; e < 4; ++e) b[e] = f2_mul(f2_mul(b[e], r2), w[e]);
            }
            if (map.turned) {
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const uint64_t x = a[e], y = b[e];
                    a[e] = f2_fma(x, c[e], f2_negate(f2_mul(y, s[e])));
                    b[e] = f2_fma(y, c[e], f2_mul(x, s[e]));
                }
            }
            if (head < (is_q ? p.num_q_heads : p.num_kv_heads)) {
                Elem* dst = (is_q ? static_cast<Elem*>(p.q_out) + token * p.q_out_stride : static_cast<Elem*>(p.k_out) + token * p.k_out_stride) + head * D;
                T::store(dst + map.off_a, a, p.wide);
                T::store(dst + map.off_b, b, p.wide);
            }
        }
#pragma unroll
        for (int i = 0; i < kUnroll; ++i) {
            now[i][0] = next[i][0];
            now[i][1] = next[i][1];
        }
    }
}

// Backward.  The warps stride over (token, part) tasks.  Their sums of the weight gradient stay with them: those of q in
// registers, those of k (a fraction of the rows) in shared memory, a lane's own 16 values each.  A CTA leaves one partial
// row per tensor, which dw_reduce_kernel adds up in a fixed order: the same result from run to run.
template <class T, int D, bool kNorm>
__global__ void __launch_bounds__(kWarps * 32, 4) qk_rope_bwd_kernel(const __grid_constant__ Params p) {
    typedef LaneMap<D> Map;
    typedef typename T::Elem Elem;
    __shared__ __align__(16) float2 cs_all[kWarps][kMaxPairs];
    __shared__ __align__(16) float weight[kNorm ? 2 : 1][D];
    __shared__ ulonglong2 dwk_all[kNorm ? kWarps : 1][4][32];  // [warp][quarter of the lane's 16 values][lane]
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const Map map(lane, p.rot);
    const int64_t n_tasks = p.n_tokens * p.warps_per_token;
    uint64_t dwq[2][4];
#pragma unroll
    for (int i = 0; i < 4; ++i) dwq[0][i] = dwq[1][i] = 0ull;
    if (kNorm) {
#pragma unroll
        for (int i = 0; i < 4; ++i) dwk_all[warp][i][lane] = make_ulonglong2(0ull, 0ull);
        stage_weights<T, D>(p, weight);
    }
    for (int64_t task = static_cast<int64_t>(blockIdx.x) * kWarps + warp; task < n_tasks;
         task += static_cast<int64_t>(gridDim.x) * kWarps) {
        const int64_t token = task / p.warps_per_token;
        const int32_t u_begin = static_cast<int32_t>(task - token * p.warps_per_token) * p.units_per_warp;
        const int32_t u_end = min(p.units, u_begin + p.units_per_warp);
        const Elem* const q = static_cast<const Elem*>(p.q) + token * p.q_stride;
        const Elem* const k = static_cast<const Elem*>(p.k) + token * p.k_stride;
        const float* const dq = p.dq + token * p.num_q_heads * D;
        const float* const dk = p.dk + token * p.num_kv_heads * D;
        struct Batch {
            typename T::Raw x[2];
            F32::Raw g[2];
        } now, next;
        auto load = [&](Batch& r, int32_t u) {
            const bool is_q = u < p.units_q;
            const int32_t head = (u - (is_q ? 0 : p.units_q)) * Map::kRows + map.row;
            const bool there = u < u_end && head < (is_q ? p.num_q_heads : p.num_kv_heads);
            const Elem* x = (is_q ? q : k) + head * D;
            const float* g = (is_q ? dq : dk) + head * D;
            r.g[0] = there ? F32::load(g + map.off_a, p.wide) : F32::zero();
            r.g[1] = there ? F32::load(g + map.off_b, p.wide) : F32::zero();
            if (kNorm) {
                r.x[0] = there ? T::load(x + map.off_a, p.wide) : T::zero();
                r.x[1] = there ? T::load(x + map.off_b, p.wide) : T::zero();
            }
        };
        load(now, u_begin);
        __syncwarp();  // the previous task's angles have been read
        token_angles(p, token, lane, cs_all[warp]);
        for (int32_t u = u_begin; u < u_end; ++u) {
            load(next, u + 1);
            const bool is_q = u < p.units_q;
            const int32_t head = (u - (is_q ? 0 : p.units_q)) * Map::kRows + map.row;
            const bool there = head < (is_q ? p.num_q_heads : p.num_kv_heads);
            uint64_t g[4], h[4];
            F32::unpack(now.g[0], g);
            F32::unpack(now.g[1], h);
            if (map.turned) {
                uint64_t c[4], s[4];
                read_angles(cs_all[warp], map.off_a >> 3, c, s);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const uint64_t x = g[i], y = h[i];
                    g[i] = f2_fma(x, c[i], f2_mul(y, s[i]));
                    h[i] = f2_fma(y, c[i], f2_negate(f2_mul(x, s[i])));
                }
            }
            if (kNorm) {
                uint64_t a[4], b[4], gw[4], hw[4];
                T::unpack(now.x[0], a);
                T::unpack(now.x[1], b);
                read_weights<D>(weight[is_q ? 0 : 1], map.off_a >> 3, gw);
                read_weights<D>(weight[is_q ? 0 : 1], map.off_b >> 3, hw);
                uint64_t ss = 0ull, st = 0ull, dot = 0ull, dou = 0ull;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    gw[i] = f2_mul(g[i], gw[i]);
                    hw[i] = f2_mul(h[i], hw[i]);
                    ss = f2_fma(a[i], a[i], ss);
                    st = f2_fma(b[i], b[i], st);
                    dot = f2_fma(gw[i], a[i], dot);
                    dou = f2_fma(hw[i], b[i], dou);
                }
                const float sum = row_sum<Map::kLanes>(f2_sum(f2_add(ss, st))), prod = row_sum<Map::kLanes>(f2_sum(f2_add(dot, dou)));
                // a row past the last head has zero gradient and adds nothing; its r is not used (eps may be 0)
                const float r = there ? rsqrtf(sum * (1.f / D) + p.eps) : 0.f;
                const float m = prod * r * (1.f / D);  // mean(g w u)
                const uint64_t r2 = f2_pack(r, r), m2 = f2_pack(-m, -m);
#pragma unroll
                for (int i = 0; i < 4; ++i) {  // a, b become u; g, h what the row adds to the weight's gradient; gw, hw dx
                    a[i] = f2_mul(a[i], r2);
                    b[i] = f2_mul(b[i], r2);
                    g[i] = f2_mul(g[i], a[i]);
                    h[i] = f2_mul(h[i], b[i]);
                    gw[i] = f2_mul(r2, f2_fma(a[i], m2, gw[i]));
                    hw[i] = f2_mul(r2, f2_fma(b[i], m2, hw[i]));
                }
                if (is_q) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        dwq[0][i] = f2_add(dwq[0][i], g[i]);
                        dwq[1][i] = f2_add(dwq[1][i], h[i]);
                    }
                } else {
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        ulonglong2 v = dwk_all[warp][i][lane];
                        v.x = f2_add(v.x, i < 2 ? g[2 * i] : h[2 * (i - 2)]);
                        v.y = f2_add(v.y, i < 2 ? g[2 * i + 1] : h[2 * (i - 2) + 1]);
                        dwk_all[warp][i][lane] = v;
                    }
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    g[i] = gw[i];
                    h[i] = hw[i];
                }
            }
            if (there) {
                Elem* dst = (is_q ? static_cast<Elem*>(p.q_out) + token * p.q_out_stride : static_cast<Elem*>(p.k_out) + token * p.k_out_stride) + head * D;
                T::store(dst + map.off_a, g, p.wide);
                T::store(dst + map.off_b, h, p.wide);
            }
            now = next;
        }
    }
    if (kNorm && p.dw_partial != nullptr) {
        __shared__ float dw_all[kNorm ? kWarps : 1][2][D];
        // over the rows of the warp, then over the warps of the CTA
#pragma unroll
        for (int t = 0; t < 2; ++t) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float* own = reinterpret_cast<const float*>(&dwk_all[warp][0][lane]);
                float x = own[(i / 4) * 128 + i % 4], y = own[(2 + i / 4) * 128 + i % 4];
                if (t == 0) {
                    float lo, hi;
                    f2_unpack(dwq[0][i / 2], lo, hi);
                    x = i & 1 ? hi : lo;
                    f2_unpack(dwq[1][i / 2], lo, hi);
                    y = i & 1 ? hi : lo;
                }
#pragma unroll
                for (int off = Map::kLanes; off < 32; off <<= 1) {
                    x += __shfl_xor_sync(0xffffffffu, x, off);
                    y += __shfl_xor_sync(0xffffffffu, y, off);
                }
                if (map.row == 0) {
                    dw_all[warp][t][map.off_a + i] = x;
                    dw_all[warp][t][map.off_b + i] = y;
                }
            }
        }
        __syncthreads();
        for (int i = threadIdx.x; i < 2 * D; i += kWarps * 32) {
            float x = 0.f;
#pragma unroll
            for (int w = 0; w < kWarps; ++w) x += dw_all[w][i / D][i % D];
            p.dw_partial[static_cast<int64_t>(blockIdx.x) * 2 * D + i] = x;
        }
    }
}

// dw[t][i] (+)= sum over the CTAs' partials, in 64 bits: one warp per column.
__global__ void dw_reduce_kernel(const float* __restrict__ partial, int n, int d, float* dq_weight, float* dk_weight, int accumulate) {
    const int col = (blockIdx.x * blockDim.x + threadIdx.x) >> 5, lane = threadIdx.x & 31;
    if (col >= 2 * d) return;
    double x = 0.0;
    for (int i = lane; i < n; i += 32) x += static_cast<double>(partial[static_cast<int64_t>(i) * 2 * d + col]);
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) x += __shfl_xor_sync(0xffffffffu, x, off);
    float* dst = col < d ? dq_weight + col : dk_weight + (col - d);
    if (lane == 0) *dst = accumulate ? static_cast<float>(static_cast<double>(*dst) + x) : static_cast<float>(x);
}

// Units per warp: a token's heads are spread over several warps only while the tokens alone do not fill the SMs (16 warps
// each), because every warp works out its token's angles again.
void split_heads(Params& p, int head_dim, int sms) {
    const int rows = 32 / (head_dim / 16);
    p.units_q = (p.num_q_heads + rows - 1) / rows;
    p.units = p.units_q + (p.num_kv_heads + rows - 1) / rows;
    int64_t want = p.n_tokens > 0 ? (static_cast<int64_t>(sms) * 16 + p.n_tokens - 1) / p.n_tokens : 1;
    if (want > p.units) want = p.units;
    p.units_per_warp = static_cast<int32_t>((p.units + want - 1) / want);
    p.warps_per_token = (p.units + p.units_per_warp - 1) / p.units_per_warp;
}

template <class T, int D>
rpx_status_t launch_forward(const Params& p, cudaStream_t stream) {
    const int64_t blocks = (p.n_tokens * p.warps_per_token + kWarps - 1) / kWarps;
    if (blocks > INT32_MAX) return RPX_ERR_SHAPE;
    if (p.q_weight != nullptr) qk_rope_kernel<T, D, true><<<static_cast<unsigned>(blocks), kWarps * 32, 0, stream>>>(p);
    else qk_rope_kernel<T, D, false><<<static_cast<unsigned>(blocks), kWarps * 32, 0, stream>>>(p);
    return cudaGetLastError() == cudaSuccess ? RPX_OK : RPX_ERR_CUDA;
}

template <class T, int D>
rpx_status_t launch_backward(const Params& p, const RopeArgs& a, int sms) {
    int64_t blocks = (p.n_tokens * p.warps_per_token + kWarps - 1) / kWarps;
    const int64_t cap = static_cast<int64_t>(sms) * kRopeBwdCtasPerSm;
    if (blocks > cap) blocks = cap;
    if (p.q_weight == nullptr) {
        qk_rope_bwd_kernel<T, D, false><<<static_cast<unsigned>(blocks), kWarps * 32, 0, a.stream>>>(p);
        return cudaGetLastError() == cudaSuccess ? RPX_OK : RPX_ERR_CUDA;
    }
    if (blocks > 0) qk_rope_bwd_kernel<T, D, true><<<static_cast<unsigned>(blocks), kWarps * 32, 0, a.stream>>>(p);
    if (cudaGetLastError() != cudaSuccess) return RPX_ERR_CUDA;
    if (p.dw_partial == nullptr) return RPX_OK;
    dw_reduce_kernel<<<2 * D / 8, 256, 0, a.stream>>>(p.dw_partial, static_cast<int>(blocks), D, a.dq_weight, a.dk_weight,
                                                      a.accumulate_dw ? 1 : 0);
    return cudaGetLastError() == cudaSuccess ? RPX_OK : RPX_ERR_CUDA;
}

}  // namespace

namespace {

Params make_params(const RopeArgs& a, int sms) {
    Params p;
    p.q = a.q;
    p.k = a.k;
    p.q_out = a.q_out;
    p.k_out = a.k_out;
    p.q_stride = a.q_tok_stride;
    p.k_stride = a.k_tok_stride;
    p.q_out_stride = a.q_out_tok_stride;
    p.k_out_stride = a.k_out_tok_stride;
    p.q_weight = a.q_weight;
    p.k_weight = a.k_weight;
    p.positions = a.positions;
    p.pos_stride = a.pos_axis_stride;
    p.inv_freq = a.inv_freq;
    p.n_tokens = a.n_tokens;
    p.num_q_heads = a.desc->num_q_heads;
    p.num_kv_heads = a.desc->num_kv_heads;
    p.rot = a.desc->rot_dim;
    p.eps = a.desc->eps;
    p.dq = a.dq;
    p.dk = a.dk;
    p.wide = true;
    for (const void* t : {a.q, a.k, static_cast<const void*>(a.q_out), static_cast<const void*>(a.k_out), static_cast<const void*>(a.dq),
                          static_cast<const void*>(a.dk)})
        p.wide = p.wide && (reinterpret_cast<uintptr_t>(t) & 31u) == 0;
    p.dw_partial = a.dq_weight != nullptr ? static_cast<float*>(a.workspace) : nullptr;
    for (int i = 0; i < kMaxPairs; ++i)
        p.axis[i] = a.desc->pair_axis != nullptr && i < p.rot / 2 ? a.desc->pair_axis[i] : 0;
    split_heads(p, a.desc->head_dim, sms);
    return p;
}

}  // namespace

size_t rope_backward_workspace(int32_t head_dim) {
    return static_cast<size_t>(kRopeBwdMaxCtas) * 2 * head_dim * sizeof(float);
}

rpx_status_t launch_qk_rope(const RopeArgs& a) {
    const int sms = sm_count();
    if (sms <= 0) return RPX_ERR_CUDA;
    const Params p = make_params(a, sms);
    const bool bf16 = a.desc->dtype == RPX_BF16;
    if (a.desc->head_dim == 128) return bf16 ? launch_forward<Bf16, 128>(p, a.stream) : launch_forward<F32, 128>(p, a.stream);
    return bf16 ? launch_forward<Bf16, 64>(p, a.stream) : launch_forward<F32, 64>(p, a.stream);
}

rpx_status_t launch_qk_rope_backward(const RopeArgs& a) {
    int sms = sm_count();
    if (sms <= 0) return RPX_ERR_CUDA;
    if (sms > kRopeBwdMaxCtas / kRopeBwdCtasPerSm) sms = kRopeBwdMaxCtas / kRopeBwdCtasPerSm;
    const Params p = make_params(a, sms);
    const bool bf16 = a.desc->dtype == RPX_BF16;
    if (a.desc->head_dim == 128) return bf16 ? launch_backward<Bf16, 128>(p, a, sms) : launch_backward<F32, 128>(p, a, sms);
    return bf16 ? launch_backward<Bf16, 64>(p, a, sms) : launch_backward<F32, 64>(p, a, sms);
}

}  // namespace rpx
