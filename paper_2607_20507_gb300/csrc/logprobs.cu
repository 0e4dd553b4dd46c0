// logprobs.cu -- log probabilities of given tokens, the entropy and the top
// alternatives of their rows (cs_logprobs).
//
// One CTA per row: the maximum; the sums S = sum w and U = sum w ln w of the
// weights w = exp((z - max) / T); then the alternatives one after another, each
// the largest logit below the one before it (ties by id).
#include "cs_internal.h"
#include "cs_device.cuh"

namespace cs {
namespace {

constexpr int kThreads = 256;

struct LogprobParams {
    const void* logits;
    const int32_t* tokens;
    float* logprob;
    float* entropy;
    int32_t* top_tokens;
    float* top_logprobs;
    int V, n_top;
    long long stride;
    float c_hi, c_lo;            // log2(e) / T
    float i_hi, i_lo;            // 1 / T
    float d_min;                 // weights of logits further below the maximum are 0
};

template <bool kF32>
__device__ __forceinline__ float logit(const void* row, int v) {
    if constexpr (kF32) return __ldcg(static_cast<const float*>(row) + v);
    else return bf16_bits_to_float(__ldcg(static_cast<const uint16_t*>(row) + v));
}

// A logit and its id as one number: the larger logit, then the lower id, is the larger.
__device__ __forceinline__ unsigned long long key_of(float z, int v) {
    const uint32_t b = __float_as_uint(z + 0.f);   // (-0 is 0)
    return (unsigned long long)(b & 0x80000000u ? ~b : b | 0x80000000u) << 32 | (uint32_t)~v;
}

template <typename T, typename F>
__device__ __forceinline__ T block_reduce(T v, T* s, F f) {
    for (int off = 16; off > 0; off >>= 1) v = f(v, __shfl_xor_sync(0xffffffffu, v, off));
    __syncthreads();
    if ((threadIdx.x & 31) == 0) s[threadIdx.x >> 5] = v;
    __syncthreads();
    T r = s[0];
    for (int w = 1; w < kThreads / 32; ++w) r = f(r, s[w]);
    return r;
}

template <bool kF32>
__global__ void __launch_bounds__(kThreads) logprobs_kernel(const LogprobParams p) {
    __shared__ unsigned long long s_red[kThreads / 32];
    const int r = blockIdx.x;
    wait_prior_grid();
    allow_dependent_launch();
    const void* row = static_cast<const char*>(p.logits) + (size_t)r * p.stride * (kF32 ? 4 : 2);
    const int tok = __ldcg(p.tokens + r);
    float* s_f = reinterpret_cast<float*>(s_red);
    float m = kNegInf;
    if (tok >= 0)
        for (int v = threadIdx.x; v < p.V; v += kThreads) m = fmaxf(m, logit<kF32>(row, v));
    m = block_reduce(m, s_f, [](float a, float b) { return fmaxf(a, b); });
    if (m == kNegInf) {   // not wanted, or nothing but masked tokens
        if (threadIdx.x == 0) {
            p.logprob[r] = kNegInf;
            if (p.entropy) p.entropy[r] = 0.f;
        }
        if (threadIdx.x < p.n_top) {
            p.top_tokens[(size_t)r * p.n_top + threadIdx.x] = -1;
            p.top_logprobs[(size_t)r * p.n_top + threadIdx.x] = kNegInf;
        }
        return;
    }
    float S = 0.f, U = 0.f;
    for (int v = threadIdx.x; v < p.V; v += kThreads) {
        const float d = fmaxf(logit<kF32>(row, v) - m, p.d_min), w = ex2_scaled(d, p.c_hi, p.c_lo);
        S += w;
        U = fmaf(w, d, U);
    }
    S = block_reduce(S, s_f, [](float a, float b) { return a + b; });
    U = block_reduce(U, s_f, [](float a, float b) { return a + b; });
    const float lse = lg2(S) * kLn2;
    auto lp = [&](float z) {
        const float d = z - m;   // (-inf where the difference, or d / T, passes fp32)
        return d * p.i_hi == kNegInf ? kNegInf : fmaf(d, p.i_hi, fmaf(d, p.i_lo, -lse));
    };
    if (threadIdx.x == 0) {
        p.logprob[r] = tok < p.V ? lp(logit<kF32>(row, tok)) : kNegInf;
        if (p.entropy) p.entropy[r] = fmaxf(0.f, lse - U / S * p.i_hi);
    }
    unsigned long long last = ~0ull;
    for (int j = 0; j < p.n_top; ++j) {
        unsigned long long best = 0;
        for (int v = threadIdx.x; v < p.V; v += kThreads) {
            const float z = logit<kF32>(row, v);
            const unsigned long long k = z == kNegInf ? 0 : key_of(z, v);
            if (k < last && k > best) best = k;
        }
        best = block_reduce(best, s_red, [](unsigned long long a, unsigned long long b) { return a > b ? a : b; });
        if (threadIdx.x == 0) {
            const int id = best ? (int)~(uint32_t)best : -1;
            p.top_tokens[(size_t)r * p.n_top + j] = id;
            p.top_logprobs[(size_t)r * p.n_top + j] = best ? lp(logit<kF32>(row, id)) : kNegInf;
        }
        last = best;
    }
}

}  // namespace

cs_status launch_logprobs(const cs_logprob_dims& d, const void* logits, const int32_t* tokens, float temperature,
                          float* out_logprob, float* out_entropy, int32_t* out_top_tokens, float* out_top_logprobs,
                          cudaStream_t stream) {
    LogprobParams p{};
    p.logits = logits;
    p.tokens = tokens;
    p.logprob = out_logprob;
    p.entropy = out_entropy;
    p.top_tokens = out_top_tokens;
    p.top_logprobs = out_top_logprobs;
    p.V = d.vocab;
    p.n_top = d.n_top;
    p.stride = d.row_stride;
    // (below 1e-37 a temperature picks the largest logits alone, as 1e-37 does)
    const double i = 1.0 / (double)(temperature < 1e-37f ? 1e-37f : temperature), c = 1.4426950408889634073599 * i;
    p.i_hi = (float)i;
    p.i_lo = (float)(i - (double)p.i_hi);
    p.c_hi = (float)c;
    p.c_lo = (float)(c - (double)p.c_hi);
    p.d_min = (float)(-300.0 / c);
    const cudaError_t e = launch_dependent(d.logit_dtype == CS_F32 ? logprobs_kernel<true> : logprobs_kernel<false>,
                                           dim3(d.rows), dim3(kThreads), 0, stream, p);
    return e == cudaSuccess ? CS_OK : cuda_fail(e, "logprobs_kernel launch");
}

}  // namespace cs
