// Clipped policy loss with a KL term over packed response log-probs, and its gradient.
//
//   d = l - o per token, or its mean over the counted tokens of the sequence;  r = e^d
//   policy = -A r, held at -A (1 + high) where A > 0 and r is above, at -A (1 - low) where A < 0 and r is below, and at
//   -A dual where A < 0 and r is above that;  kl = l - f, (l - f)^2 / 2 or e^(f - l) - (f - l) - 1
//   loss = sum w (policy + b kl),   dl = upstream w (-A r where not held + b dkl/dl)
//
// d policy / d l is -A r under both kinds of ratio: with the sequence's ratio every counted token's policy term holds the
// same r, and n terms of weight w with dr/dl = r / n each add up to the one w r.
//
// Bound by memory in principle (at most 21 bytes a token: l, o, f, mask, an advantage, dl) and by launches in truth: the
// weights need the counts of all sequences first.  So batches of up to kSmallTokens tokens in up to kSmallBatch sequences (a warp
// each) are one launch of one CTA, larger ones two: one CTA per sequence counts (and takes the mean of d), and the pass over the
// tokens is launched on top of it with its first tokens already on their way; its last CTA adds up the CTAs' sums.
//
// Measured: 8 x 250 tokens 5.4 us, 256 ragged sequences of up to 2048 10 us, 1024 of up to 4096 with every input (2.3 M
// tokens) 28 us, 27 % of the copy bandwidth: the chains of some 100 instructions a token.  A lane has four tokens at a time and a
// warp's tokens follow one another, so that a sequence is looked up, and its weight divided, where one begins.
#include "rpx_internal.h"
#include "rpx_ptx.cuh"

namespace rpx {

namespace {

constexpr int kThreads = 256, kSmallThreads = 512;
// One CTA (of 512 threads, four tokens each: with 1024 it spills, 7.1 us for 5.8) against two launches, 8 x 250 tokens: 5.8 us in a
// graph for 7.6, and 16.2 for 18.4 a call from Python; masked 6.3 for 7.8, 32 x 60 6.8 for 7.9, one sequence of 2000 7.4 for 7.7.
// Beyond, the one CTA loses (with 1024 threads): 8 x 1024 masked 12.2 us for 7.5; 48 x 41 9.4 for 9.1, 400 x 2 17.3 for 9.6, 8192 x
// 1 208 for 22.
constexpr int64_t kSmallTokens = 2048;
constexpr int32_t kSmallBatch = 32;
constexpr int kCtasPerSm = 3;  // (four, with 64 registers, spill: 31 us for 28)
constexpr int kSums = 4;  // policy, kl, clipped, ratio

struct Params {
    const float *l, *o, *f, *adv;  // o, f nullable
    const uint8_t* mask;           // nullable
    const int32_t* cu;
    int32_t batch, n_tokens;
    const float* upstream;         // nullable
    float *stats, *dl;             // dl nullable
    int32_t kl;
    int32_t steps, more;           // 128 tokens each: of every warp, and the first warps that have one more
    bool by_sequence, sequence_mean, adv_per_token, zero_rest, wide;  // wide: all token arrays allow 16-byte (mask: 4-byte) accesses
    double log_low, log_high, log_dual;  // borders of d
    float near_low, near_high, near_dual;  // rounded
    float low, high, dual;               // what r is held at
    float kl_coef;
    double kl_coef64, count;
    int32_t* seq_n;                // workspace [batch]: counted tokens
    double* seq_d;                 // workspace [batch]: mean of d (sequence ratio)
    double* partial;               // workspace [CTAs][kSums]
    uint32_t* ticket;              // workspace
    int32_t* status;
};

__device__ __forceinline__ double warp_sum(double x) {
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) x += __shfl_xor_sync(0xffffffffu, x, off);
    return x;
}

// Bounds of a sequence; one that does not fit is empty.
__device__ __forceinline__ bool sequence(const Params& p, int32_t s, int32_t* begin, int32_t* end) {
    *begin = __ldg(p.cu + s);
    *end = __ldg(p.cu + s + 1);
    return *begin >= 0 && *begin <= *end && *end <= p.n_tokens;
}

__device__ __forceinline__ void count_one(const Params& p, int64_t t, bool with_d, int32_t* n, double* d) {
    if (p.mask != nullptr && __ldg(p.mask + t) == 0) return;
    *n += 1;
    if (with_d) *d += static_cast<double>(__ldg(p.l + t)) - static_cast<double>(__ldg(p.o + t));
}

// Counted tokens of a sequence and the sum of their d, as one of `lanes` threads sees them.
__device__ __forceinline__ void count_tokens(const Params& p, int32_t begin, int32_t end, int lane, int lanes, int32_t* n, double* d) {
    *n = 0;
    *d = 0.0;
    if (p.mask == nullptr && !p.by_sequence) {
        if (lane == 0) *n = end - begin;
        return;
    }
    const bool with_d = p.by_sequence && p.o != nullptr;
    if (p.wide) {  // by fours
#pragma unroll 4
        for (int64_t t = static_cast<int64_t>(begin & ~3) + 4 * lane; t < end; t += 4 * lanes) {  // (up to 2^31 tokens: 64 bits before the sum)
            if (t + 4 > p.n_tokens) {
                for (int64_t u = t < begin ? begin : t; u < end; ++u) count_one(p, u, with_d, n, d);
                continue;
            }
            uint32_t m = p.mask != nullptr ? __ldg(reinterpret_cast<const uint32_t*>(p.mask + t)) : ~0u;
            float4 l, o;
            if (with_d) {
                l = __ldg(reinterpret_cast<const float4*>(p.l + t));
                o = __ldg(reinterpret_cast<const float4*>(p.o + t));
            }
            if (t < begin) m &= ~0u << 8 * (begin - t);
            if (t + 4 > end) m &= ~0u >> 8 * (t + 4 - end);
            *n += __popc(__vcmpgtu4(m, 0u)) >> 3;
            if (with_d) {
                *d += (m & 255u) != 0u ? static_cast<double>(l.x) - static_cast<double>(o.x) : 0.0;
                *d += (m & 0xff00u) != 0u ? static_cast<double>(l.y) - static_cast<double>(o.y) : 0.0;
                *d += (m & 0xff0000u) != 0u ? static_cast<double>(l.z) - static_cast<double>(o.z) : 0.0;
                *d += (m >> 24) != 0u ? static_cast<double>(l.w) - static_cast<double>(o.w) : 0.0;
            }
        }
        return;
    }
#pragma unroll 4
    for (int64_t t = static_cast<int64_t>(begin) + lane; t < end; t += lanes) count_one(p, t, with_d, n, d);
}

// (Five CTAs an SM: with the 60 registers that the compiler may take otherwise, 256 ragged sequences take 10.8 us for 9.9.)
__global__ void __launch_bounds__(kThreads, 5) policy_count_kernel(const __grid_constant__ Params p) {
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    __shared__ int32_t part_n[kThreads / 32];
    __shared__ double part_d[kThreads / 32];
    if (blockIdx.x == 0 && threadIdx.x == 0) *p.ticket = 0u;
    for (int32_t s = blockIdx.x; s < p.batch; s += gridDim.x) {
        int32_t begin, end, n;
        double d;
        if (!sequence(p, s, &begin, &end)) {
            if (threadIdx.x == 0 && p.status != nullptr) atomicCAS(p.status, 0, RPX_ERR_DEVICE_DATA);
            begin = end = 0;
        }
        count_tokens(p, begin, end, threadIdx.x, kThreads, &n, &d);
        n = __reduce_add_sync(0xffffffffu, n);
        if (p.by_sequence) d = warp_sum(d);
        if ((threadIdx.x & 31) == 0) {
            part_n[threadIdx.x >> 5] = n;
            part_d[threadIdx.x >> 5] = d;
        }
        __syncthreads();
        if (threadIdx.x == 0) {
            for (int w = 1; w < kThreads / 32; ++w) {
                n += part_n[w];
                d += part_d[w];
            }
            p.seq_n[s] = n;
            if (p.by_sequence) p.seq_d[s] = n > 0 ? d / n : 0.0;
        }
        __syncthreads();
    }
}

// e^x, e^x - 1 and e^x - 1 - x together: x = n ln 2 + g with |g| <= ln 2 / 2 (the reduction of Cody and Waite: ln 2 in two parts,
// n times the first exact), q = e^g - 1 by its Taylor polynomial of degree 8 (what is left out is below 2^-32), e^x = 2^n (1 + q).
// Where n is 0 neither e^x - 1 nor e^x - 1 - x has lost anything; elsewhere both are as large as their parts.  2 to 3 roundings, no
// branch, NaN kept, infinity above the largest value, 0 from n = -126 on: below 2^-125.5, x < -86.99, where 2^n / 2 is none of
// float32's normal numbers.  (The fast e^x that this library is compiled with is four times as far
// off; expm1f, called for each, took a third of the kernel's time.)
struct Exp {
    float exp, minus_one, minus_linear;
};
__device__ __forceinline__ Exp exponentials(float x) {
    float y;
    asm("{\n\t.reg .f32 t;\n\tmin.NaN.f32 t, %1, 0f42B20000;\n\tmax.NaN.f32 %0, t, 0fC2AF0000;\n\t}" : "=f"(y) : "f"(x));  // [-87.5, 89]
    const float shifted = fmaf(y, 1.44269504f, 12582912.f);  // 1.5 * 2^23: n in the low bits
    const float n = shifted - 12582912.f;
    const float g = fmaf(n, -1.42860682e-6f, fmaf(n, -0.693145751953125f, y));
    const float half = __int_as_float((__float_as_int(shifted) << 23) + (126 << 23));  // 2^n / 2
    float a = 1.f / 40320.f;
    a = fmaf(a, g, 1.f / 5040.f);
    a = fmaf(a, g, 1.f / 720.f);
    a = fmaf(a, g, 1.f / 120.f);
    a = fmaf(a, g, 1.f / 24.f);
    a = fmaf(a, g, 1.f / 6.f);
    a = fmaf(a, g, 0.5f);
    const float rest = a * (g * g), q = g + rest;
    const float one = 1.f + q, m = fmaf(half, q, half - 0.5f);
    return {(one + one) * half, m + m, n == 0.f ? rest : (m + m) - x};
}

struct Four {
    alignas(16) float l[4], o[4], f[4], adv[4];  // (read as 16 bytes, also where they have left the registers)
    uint32_t counted;  // a bit each
};

template <int kBlock, bool kSmall>
__global__ void __launch_bounds__(kBlock, kSmall ? 1 : kCtasPerSm) policy_loss_kernel(const __grid_constant__ Params p) {
    constexpr int kWarps = kBlock / 32;
    __shared__ double part[kWarps][kSums];
    __shared__ int64_t part_n[kWarps];
    __shared__ int32_t part_s[kWarps];
    __shared__ bool last;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    auto load = [&](Four& x, int32_t t0) {
        x.counted = 0u;
        if (p.wide && t0 <= p.n_tokens - 4) {
            *reinterpret_cast<float4*>(x.l) = __ldcs(reinterpret_cast<const float4*>(p.l + t0));
            if (p.o != nullptr) *reinterpret_cast<float4*>(x.o) = __ldcs(reinterpret_cast<const float4*>(p.o + t0));
            if (p.f != nullptr) *reinterpret_cast<float4*>(x.f) = __ldcs(reinterpret_cast<const float4*>(p.f + t0));
            if (p.adv_per_token) *reinterpret_cast<float4*>(x.adv) = __ldcs(reinterpret_cast<const float4*>(p.adv + t0));
            const uint32_t m = p.mask != nullptr ? __ldcs(reinterpret_cast<const uint32_t*>(p.mask + t0)) : ~0u;
#pragma unroll
            for (int i = 0; i < 4; ++i) x.counted |= (m >> (8 * i) & 255u) != 0u ? 1u << i : 0u;
            return;
        }
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (i < p.n_tokens - t0) {
                x.l[i] = p.l[t0 + i];
                if (p.o != nullptr) x.o[i] = p.o[t0 + i];
                if (p.f != nullptr) x.f[i] = p.f[t0 + i];
                if (p.adv_per_token) x.adv[i] = p.adv[t0 + i];
                if (p.mask == nullptr || p.mask[t0 + i] != 0) x.counted |= 1u << i;
            }
    };
    // a warp's tokens follow one another, 128 a step: its lanes seldom have to look a sequence up
    const int32_t at = static_cast<int32_t>(blockIdx.x) * kWarps + warp;
    int32_t step = p.steps * at + min(at, p.more);
    const int32_t step_end = step + p.steps + (at < p.more ? 1 : 0);
    int32_t t0 = step < step_end ? step * 128 + lane * 4 : p.n_tokens;  // (at most 2^31 - 4)
    Four now;
    if (t0 < p.n_tokens) load(now, t0);

    // ---- counts: of this CTA's own making, or of the kernel before
    if constexpr (kSmall) {
        for (int32_t s = warp; s < p.batch; s += kWarps) {
            int32_t begin, end, n;
            double d;
            if (!sequence(p, s, &begin, &end)) {
                if (lane == 0 && p.status != nullptr) atomicCAS(p.status, 0, RPX_ERR_DEVICE_DATA);
                begin = end = 0;
            }
            count_tokens(p, begin, end, lane, 32, &n, &d);
            n = __reduce_add_sync(0xffffffffu, n);
            if (p.by_sequence) d = warp_sum(d);
            if (lane == 0) {
                p.seq_n[s] = n;
                if (p.by_sequence) p.seq_d[s] = n > 0 ? d / n : 0.0;
            }
        }
        __syncthreads();
    } else {
        asm volatile("griddepcontrol.wait;" ::: "memory");
    }
    int64_t total = 0;
    int32_t sequences = 0;
    for (int32_t s = threadIdx.x; s < p.batch; s += kBlock) {
        const int32_t n = p.seq_n[s];
        total += n;
        sequences += n > 0 ? 1 : 0;
    }
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) total += __shfl_xor_sync(0xffffffffu, total, off);
    sequences = __reduce_add_sync(0xffffffffu, sequences);
    if (lane == 0) {
        part_n[warp] = total;
        part_s[warp] = sequences;
    }
    __syncthreads();
    total = 0;
    sequences = 0;
    for (int w = 0; w < kWarps; ++w) {
        total += part_n[w];
        sequences += part_s[w];
    }
    const double over = p.count > 0.0 ? p.count : p.sequence_mean ? static_cast<double>(sequences) : static_cast<double>(total);
    const float upstream = p.upstream != nullptr ? __ldg(p.upstream) : 1.f;

    // ---- the tokens, four a thread
    double sums[kSums] = {0.0, 0.0, 0.0, 0.0};
    int32_t s = 0, s_hi = 0, begin = 0, end = 0;  // the sequence whose numbers are at hand
    bool fits = false;
    double w = 0.0, d_seq = 0.0;
    float a_seq = 0.f, w_up = 0.f;  // (w_up: w times the upstream gradient)
    for (; step < step_end; ++step, t0 = step < step_end ? t0 + 128 : t0) {  // (128 more than the last ones may not fit 32 bits)
        Four next;
        if (step + 1 < step_end && t0 < p.n_tokens - 128) load(next, t0 + 128);
        const bool alone = __all_sync(0xffffffffu, fits && t0 <= end - 4);  // every lane stays in its sequence
        if (!alone) {
            // sequences of the warp's first and last token
            const int32_t first = step * 128;
            s = s_hi = last_at_or_before(p.cu, p.batch, first, lane);
            const int32_t rest = min(127, p.n_tokens - 1 - first);
            if (__ldg(p.cu + s + 1) <= first + rest) s_hi = last_at_or_before(p.cu, p.batch, first + rest, lane);
            // the thread's first token, among these
            int32_t up = s_hi + 1;
            while (up - s > 1) {
                const int32_t mid = s + (up - s) / 2;
                if (__ldg(p.cu + mid) <= t0) s = mid;
                else up = mid;
            }
            fits = false;
        }
        if (t0 < p.n_tokens) {
            float grads[4];
            double policy = 0.0, ratio = 0.0, kl_sum = 0.0;  // sums of tokens of one weight
            int clips = 0;
            uint32_t written = 0u;
            auto add = [&] {
                sums[0] += w * policy;
                sums[1] += w * kl_sum;
                sums[2] += w * clips;
                sums[3] += w * ratio;
            };
            auto token = [&](int i) {
                const bool counted = (now.counted >> i & 1u) != 0u;
                const float a = p.adv_per_token ? now.adv[i] : a_seq;
                const float d = p.by_sequence ? static_cast<float>(d_seq) : p.o != nullptr ? now.l[i] - now.o[i] : 0.f;
                bool above = d > p.near_high, below = d < p.near_low, far = d > p.near_dual;
                if (d == p.near_high || d == p.near_low || d == p.near_dual) {  // the rounding of d decides nothing
                    const double exact = p.by_sequence ? d_seq : p.o != nullptr ? static_cast<double>(now.l[i]) - static_cast<double>(now.o[i]) : 0.0;
                    above = exact > p.log_high;
                    below = exact < p.log_low;
                    far = exact > p.log_dual;
                }
                const float r = exponentials(d).exp;
                const bool clipped = a > 0.f ? above : a < 0.f && (below || far);
                const float held = a > 0.f ? p.high : below ? p.low : p.dual;
                float g = clipped ? 0.f : -a * r;
                policy += counted ? static_cast<double>(-a * (clipped ? held : r)) : 0.0;
                ratio += counted ? static_cast<double>(r) : 0.0;
                clips += counted && clipped ? 1 : 0;
                if (p.kl != 0) {
                    const float x = now.f[i] - now.l[i];
                    float kl = -x, slope = 1.f;
                    if (p.kl == 2) {
                        kl = 0.5f * x * x;
                        slope = -x;
                    } else if (p.kl == 3) {
                        const Exp e = exponentials(x);
                        kl = e.minus_linear;
                        slope = -e.minus_one;
                    }
                    kl_sum += counted ? static_cast<double>(kl) : 0.0;
                    g += p.kl_coef * slope;
                }
                grads[i] = counted ? g * w_up : 0.f;
            };
            if (alone) {
                written = 15u;
#pragma unroll
                for (int i = 0; i < 4; ++i) token(i);
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int32_t t = t0 + i;
                    if (!fits || t >= end) {
                        if (i > 0) {
                            add();
                            policy = ratio = kl_sum = 0.0;
                            clips = 0;
                        }
                        while (s < s_hi && __ldg(p.cu + s + 1) <= t) ++s;
                        fits = sequence(p, s, &begin, &end) && begin <= t && t < end;
                        w = 0.0;
                        if (fits) {
                            const int32_t n = p.seq_n[s];
                            w = n > 0 ? 1.0 / (p.sequence_mean ? over * n : over) : 0.0;
                            if (p.by_sequence) d_seq = p.seq_d[s];
                            if (!p.adv_per_token) a_seq = __ldg(p.adv + s);
                        }
                        w_up = static_cast<float>(w) * upstream;
                    }
                    grads[i] = 0.f;
                    if (fits || p.zero_rest) written |= 1u << i;
                    if (!fits) continue;
                    token(i);
                }
            }
            add();
            if (p.dl != nullptr) {
                if (written == 15u && p.wide) {
                    *reinterpret_cast<float4*>(p.dl + t0) = make_float4(grads[0], grads[1], grads[2], grads[3]);
                } else {
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        if ((written >> i & 1u) != 0u) p.dl[t0 + i] = grads[i];
                }
            }
        }
        now = next;
    }
    // ---- the CTA's sums, and with the last CTA those of all, in order
#pragma unroll
    for (int k = 0; k < kSums; ++k) {
        const double x = warp_sum(sums[k]);
        if (lane == 0) part[warp][k] = x;
    }
    __syncthreads();
    if (threadIdx.x < kSums) {
        double x = 0.0;
        for (int w = 0; w < kWarps; ++w) x += part[w][threadIdx.x];
        if (kSmall) part[0][threadIdx.x] = x;
        else p.partial[static_cast<int64_t>(blockIdx.x) * kSums + threadIdx.x] = x;
    }
    if constexpr (!kSmall) {
        __threadfence();
        __syncthreads();
        if (threadIdx.x == 0) last = atomicAdd(p.ticket, 1u) + 1u == gridDim.x;
        __syncthreads();
        if (!last) return;
        __threadfence();
        if (warp < kSums) {  // a warp a sum
            double x = 0.0;
            for (uint32_t b = lane; b < gridDim.x; b += 32) x += __ldcg(p.partial + static_cast<int64_t>(b) * kSums + warp);
            x = warp_sum(x);
            if (lane == 0) part[0][warp] = x;
        }
    }
    __syncthreads();
    if (threadIdx.x == 0) {
        p.stats[0] = static_cast<float>(part[0][0] + p.kl_coef64 * part[0][1]);
        p.stats[1] = static_cast<float>(part[0][0]);
        p.stats[2] = static_cast<float>(part[0][1]);
        p.stats[3] = static_cast<float>(part[0][2]);
        p.stats[4] = static_cast<float>(part[0][3]);
        p.stats[5] = static_cast<float>(total);
    }
}

size_t counts_bytes(int32_t batch) { return align_up(static_cast<size_t>(batch) * sizeof(int32_t), 256); }
size_t means_bytes(int32_t batch) { return align_up(static_cast<size_t>(batch) * sizeof(double), 256); }
constexpr int kMaxCtas = 1024;

}  // namespace

size_t policy_workspace(int32_t batch, int64_t) { return counts_bytes(batch) + means_bytes(batch) + kMaxCtas * kSums * sizeof(double) + 256; }

rpx_status_t launch_policy_loss(const PolicyArgs& a) {
    const rpx_policy_desc_t& c = *a.desc;
    if (a.batch == 0 || a.n_tokens == 0) {
        if (c.zero_rest != 0 && a.dlogprobs != nullptr && a.n_tokens > 0 &&
            cudaMemsetAsync(a.dlogprobs, 0, static_cast<size_t>(a.n_tokens) * sizeof(float), a.stream) != cudaSuccess)
            return RPX_ERR_CUDA;
        return cudaMemsetAsync(a.stats, 0, 6 * sizeof(float), a.stream) == cudaSuccess ? RPX_OK : RPX_ERR_CUDA;
    }
    Params p = {};
    p.l = a.logprobs;
    p.o = a.old_logprobs;
    p.f = a.ref_logprobs;
    p.adv = a.advantages;
    p.mask = a.mask;
    p.cu = a.cu;
    p.batch = a.batch;
    p.n_tokens = static_cast<int32_t>(a.n_tokens);  // (below 2^31 - 1)
    p.upstream = a.upstream;
    p.stats = a.stats;
    p.dl = a.dlogprobs;
    p.kl = c.kl;
    p.by_sequence = c.ratio == RPX_RATIO_SEQUENCE;
    p.sequence_mean = c.mean == RPX_MEAN_SEQUENCES;
    p.adv_per_token = c.adv_per_token != 0;
    p.zero_rest = c.zero_rest != 0;
    p.log_high = log1p(c.clip_high);
    p.log_low = log1p(-c.clip_low);
    p.log_dual = c.clip_dual > 0.0 ? log(c.clip_dual) : HUGE_VAL;
    p.near_low = static_cast<float>(p.log_low);
    p.near_high = static_cast<float>(p.log_high);
    p.near_dual = static_cast<float>(p.log_dual);
    p.high = static_cast<float>(1.0 + c.clip_high);
    p.low = static_cast<float>(1.0 - c.clip_low);
    p.dual = static_cast<float>(c.clip_dual);
    p.kl_coef64 = c.kl_coef;
    p.kl_coef = static_cast<float>(c.kl_coef);
    p.count = c.count;
    p.wide = (reinterpret_cast<uintptr_t>(a.mask) & 3u) == 0;
    for (const void* t : {static_cast<const void*>(p.l), static_cast<const void*>(p.o), static_cast<const void*>(p.f), static_cast<const void*>(p.dl),
                          static_cast<const void*>(p.adv_per_token ? p.adv : nullptr)})
        p.wide = p.wide && (reinterpret_cast<uintptr_t>(t) & 15u) == 0;
    uint8_t* ws = static_cast<uint8_t*>(a.workspace);
    p.seq_n = reinterpret_cast<int32_t*>(ws);
    ws += counts_bytes(a.batch);
    p.seq_d = reinterpret_cast<double*>(ws);
    ws += means_bytes(a.batch);
    p.partial = reinterpret_cast<double*>(ws);
    ws += kMaxCtas * kSums * sizeof(double);
    p.ticket = reinterpret_cast<uint32_t*>(ws);
    p.status = a.device_status;
    auto share_out = [&](int64_t warps) {
        const int64_t steps = (a.n_tokens + 127) / 128;
        p.steps = static_cast<int32_t>(steps / warps);
        p.more = static_cast<int32_t>(steps % warps);
    };
    if (a.n_tokens <= kSmallTokens && a.batch <= kSmallBatch) {
        share_out(kSmallThreads / 32);
        policy_loss_kernel<kSmallThreads, true><<<1, kSmallThreads, 0, a.stream>>>(p);
        return cudaGetLastError() == cudaSuccess ? RPX_OK : RPX_ERR_CUDA;
    }
    const int sms = sm_count();
    if (sms <= 0) return RPX_ERR_CUDA;
    const int32_t counters = a.batch < sms * 8 ? a.batch : sms * 8;
    policy_count_kernel<<<static_cast<unsigned>(counters), kThreads, 0, a.stream>>>(p);
    if (cudaGetLastError() != cudaSuccess) return RPX_ERR_CUDA;
    int64_t ctas = (a.n_tokens + kThreads * 4 - 1) / (kThreads * 4);
    const int64_t cap = sms * kCtasPerSm < kMaxCtas ? sms * kCtasPerSm : kMaxCtas;
    if (ctas > cap) ctas = cap;
    share_out(ctas * (kThreads / 32));
    return launch_on_top(policy_loss_kernel<kThreads, false>, static_cast<unsigned>(ctas), kThreads, 0, a.stream, p);
}

}  // namespace rpx
