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
// weights need the counts of all sequences first.  So batches of up to kSmallTokens tokens are one launch of one CTA, larger
// ones two: one CTA per sequence counts (and takes the mean of d), and the pass over the tokens is launched on top of it with
// its first tokens already on their way; its last CTA adds up the CTAs' sums.
#include "rpx_internal.h"

namespace rpx {

namespace {

constexpr int kThreads = 256, kSmallThreads = 1024;
constexpr int64_t kSmallTokens = 8192;
constexpr int kCtasPerSm = 4;
constexpr int kSums = 4;  // policy, kl, clipped, ratio

struct Params {
    const float *l, *o, *f, *adv;  // o, f nullable
    const uint8_t* mask;           // nullable
    const int32_t* cu;
    int32_t batch;
    int64_t n_tokens;
    const float* upstream;         // nullable
    float *stats, *dl;             // dl nullable
    int32_t kl;
    bool by_sequence, sequence_mean, adv_per_token, wide;  // wide: all token arrays allow 16-byte (mask: 4-byte) accesses
    double log_low, log_high, log_dual;  // borders of d
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

// Counted tokens of a sequence and the sum of their d, as one of `lanes` threads sees them.
__device__ __forceinline__ void count_tokens(const Params& p, int32_t begin, int32_t end, int lane, int lanes, int32_t* n, double* d) {
    *n = 0;
    *d = 0.0;
    if (p.mask == nullptr && !p.by_sequence) {
        if (lane == 0) *n = end - begin;
        return;
    }
#pragma unroll 4
    for (int64_t t = begin + lane; t < end; t += lanes) {
        const bool counted = p.mask == nullptr || __ldg(p.mask + t) != 0;
        *n += counted ? 1 : 0;
        if (p.by_sequence && p.o != nullptr && counted) *d += static_cast<double>(__ldg(p.l + t)) - static_cast<double>(__ldg(p.o + t));
    }
}

__global__ void __launch_bounds__(kThreads) policy_count_kernel(const __grid_constant__ Params p) {
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

// e^x from expm1 (1 ulp; the fast e^x that this library is compiled with is four times as far off): 1 + expm1(|x|) loses
// nothing, and the other side is its reciprocal.
__device__ __forceinline__ float exp_near(float x) {
    const float e = 1.f + expm1f(fabsf(x));
    return x < 0.f ? __frcp_rn(e) : e;
}
// e^x - 1 - x: its series where the terms all but cancel (the first one left out is below 2^-28 of the first one taken)
__device__ __forceinline__ float exp_minus_linear(float x) {
    if (fabsf(x) >= 0.25f) return expm1f(x) - x;
    float y = 1.f / 40320.f;
    y = fmaf(y, x, 1.f / 5040.f);
    y = fmaf(y, x, 1.f / 720.f);
    y = fmaf(y, x, 1.f / 120.f);
    y = fmaf(y, x, 1.f / 24.f);
    y = fmaf(y, x, 1.f / 6.f);
    y = fmaf(y, x, 0.5f);
    return y * x * x;
}

struct Four {
    float l[4], o[4], f[4], adv[4];
    uint32_t counted;  // a bit each
};

template <int kBlock, bool kSmall>
__global__ void __launch_bounds__(kBlock) policy_loss_kernel(const __grid_constant__ Params p) {
    constexpr int kWarps = kBlock / 32;
    __shared__ double part[kWarps][kSums];
    __shared__ int64_t part_n[kWarps];
    __shared__ int32_t part_s[kWarps];
    __shared__ bool last;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    auto load = [&](Four& x, int64_t t0) {
        x.counted = 0u;
        if (p.wide && t0 + 4 <= p.n_tokens) {
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
            if (t0 + i < p.n_tokens) {
                x.l[i] = p.l[t0 + i];
                if (p.o != nullptr) x.o[i] = p.o[t0 + i];
                if (p.f != nullptr) x.f[i] = p.f[t0 + i];
                if (p.adv_per_token) x.adv[i] = p.adv[t0 + i];
                if (p.mask == nullptr || p.mask[t0 + i] != 0) x.counted |= 1u << i;
            }
    };
    const int64_t stride = static_cast<int64_t>(gridDim.x) * kBlock * 4;
    int64_t t0 = (static_cast<int64_t>(blockIdx.x) * kBlock + threadIdx.x) * 4;
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
    for (; __any_sync(0xffffffffu, t0 < p.n_tokens); t0 += stride) {
        Four next;
        if (t0 + stride < p.n_tokens) load(next, t0 + stride);
        // sequences of the warp's first and last token: 32 offsets a step (the last one that starts at or before a token)
        auto find = [&](int64_t t) {
            int32_t lo = 0, hi = p.batch;
            while (hi - lo > 1) {
                const int32_t step = (hi - lo + 31) / 32;
                const int64_t at = lo + static_cast<int64_t>(lane) * step;
                const uint32_t before = __ballot_sync(0xffffffffu, at < hi && __ldg(p.cu + at) <= t);
                lo += (before != 0u ? 31 - __clz(static_cast<int>(before)) : 0) * step;
                hi = hi - lo > step ? lo + step : hi;
            }
            return lo;
        };
        const int64_t first = __shfl_sync(0xffffffffu, t0, 0);
        int32_t s_lo = find(first), s_hi = s_lo;
        if (__ldg(p.cu + s_lo + 1) < min(first + 128, p.n_tokens)) s_hi = find(min(first + 127, p.n_tokens - 1));
        // the thread's first token, among these
        int32_t s = s_lo, up = s_hi + 1;
        while (up - s > 1) {
            const int32_t mid = s + (up - s) / 2;
            if (__ldg(p.cu + mid) <= t0) s = mid;
            else up = mid;
        }
        if (t0 < p.n_tokens) {
            int32_t begin = 0, end = 0;  // of the sequence whose numbers are at hand
            bool fits = false;
            double w = 0.0, d_seq = 0.0;
            float a_seq = 0.f, grads[4];
            uint32_t written = 0u;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int64_t t = t0 + i;
                if (!fits || t >= end) {
                    while (s < s_hi && __ldg(p.cu + s + 1) <= t) ++s;
                    fits = sequence(p, s, &begin, &end) && begin <= t && t < end;
                    w = 0.0;
                    if (fits) {
                        const int32_t n = p.seq_n[s];
                        w = n > 0 ? 1.0 / (p.sequence_mean ? over * n : over) : 0.0;
                        if (p.by_sequence) d_seq = p.seq_d[s];
                        if (!p.adv_per_token) a_seq = __ldg(p.adv + s);
                    }
                }
                grads[i] = 0.f;
                if (t >= p.n_tokens || !fits) continue;
                written |= 1u << i;
                if ((now.counted >> i & 1u) == 0u) continue;
                const float a = p.adv_per_token ? now.adv[i] : a_seq;
                // the difference of two floats in 64 bits: on the side of a border that it is on
                const double d = p.by_sequence ? d_seq : p.o != nullptr ? static_cast<double>(now.l[i]) - static_cast<double>(now.o[i]) : 0.0;
                const float r = exp_near(static_cast<float>(d));
                float held = 0.f;
                bool clipped = false;
                if (a > 0.f && d > p.log_high) {
                    clipped = true;
                    held = p.high;
                } else if (a < 0.f && (d < p.log_low || d > p.log_dual)) {
                    clipped = true;
                    held = d < p.log_low ? p.low : p.dual;
                }
                float g = clipped ? 0.f : -a * r, kl = 0.f;
                if (p.kl != 0) {
                    const float x = now.f[i] - now.l[i];
                    kl = p.kl == 1 ? -x : p.kl == 2 ? 0.5f * x * x : exp_minus_linear(x);
                    g += p.kl_coef * (p.kl == 1 ? 1.f : p.kl == 2 ? -x : -expm1f(x));
                }
                grads[i] = static_cast<float>(w) * g * upstream;
                sums[0] += w * static_cast<double>(-a * (clipped ? held : r));
                sums[1] += w * static_cast<double>(kl);
                sums[2] += clipped ? w : 0.0;
                sums[3] += w * static_cast<double>(r);
            }
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
    if (a.batch == 0 || a.n_tokens == 0)
        return cudaMemsetAsync(a.stats, 0, 6 * sizeof(float), a.stream) == cudaSuccess ? RPX_OK : RPX_ERR_CUDA;
    const rpx_policy_desc_t& c = *a.desc;
    Params p = {};
    p.l = a.logprobs;
    p.o = a.old_logprobs;
    p.f = a.ref_logprobs;
    p.adv = a.advantages;
    p.mask = a.mask;
    p.cu = a.cu;
    p.batch = a.batch;
    p.n_tokens = a.n_tokens;
    p.upstream = a.upstream;
    p.stats = a.stats;
    p.dl = a.dlogprobs;
    p.kl = c.kl;
    p.by_sequence = c.ratio == RPX_RATIO_SEQUENCE;
    p.sequence_mean = c.mean == RPX_MEAN_SEQUENCES;
    p.adv_per_token = c.adv_per_token != 0;
    p.log_high = log1p(c.clip_high);
    p.log_low = log1p(-c.clip_low);
    p.log_dual = c.clip_dual > 0.0 ? log(c.clip_dual) : HUGE_VAL;
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
    if (a.n_tokens <= kSmallTokens) {
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
    return launch_on_top(policy_loss_kernel<kThreads, false>, static_cast<unsigned>(ctas), kThreads, 0, a.stream, p);
}

}  // namespace rpx
