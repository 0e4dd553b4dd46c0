// chunk_attention.cu -- attention of every request's newest tokens over the paged
// bf16 cache, causal among them (cs_chunk_attention; the formula is in cachespec.h).
//
// A CTA takes 32 query rows of one request and KV head (row r of a request is token
// r / G, query head h G + r % G) and passes once over their keys, 32 at a time, with
// the running maximum and sum of the softmax; four threads share a row, each 32 of
// its dims.
#include "cs_internal.h"
#include "ragged.cuh"

namespace cs {
namespace {

constexpr int kD = 128;
constexpr int kRows = 32, kKeys = 32, kThreads = 128;

struct ChunkParams {
    RaggedBatch batch;
    const __nv_bfloat16 *q, *k_pages, *v_pages;
    const int32_t* page_table;
    __nv_bfloat16* out;
    int64_t q_stride;
    int Hq, Hkv, G, ps_log2, max_pages, P;
    float scale_log2;
};

__global__ void __launch_bounds__(kThreads) chunk_attention_kernel(const ChunkParams p) {
    __shared__ float sk[kKeys][kD + 4], sv[kKeys][kD + 4];
    __shared__ int s_b, s_block;
    wait_prior_grid();
    allow_dependent_launch();
    if (threadIdx.x == 0) {
        long long left = blockIdx.x;
        int b = 0;
        for (; b < p.batch.B; ++b) {
            int start, n, L;
            p.batch.rows_of(b, start, n, L);
            const long long blocks = ((long long)n * p.G + kRows - 1) / kRows;
            if (left < blocks) break;
            left -= blocks;
        }
        s_b = b;
        s_block = (int)left;
    }
    __syncthreads();
    const int b = s_b, h = blockIdx.y;
    if (b >= p.batch.B) return;
    int start, n, L;
    p.batch.rows_of(b, start, n, L);
    const int r = s_block * kRows + (int)threadIdx.x / 4, part = threadIdx.x & 3;
    const int i = min(r / p.G, n - 1), g = r % p.G;
    const bool live = r < n * p.G;
    const int last_i = min((s_block * kRows + kRows - 1) / p.G, n - 1);
    const int seen = L - n + i + 1, most = L - n + last_i + 1;   // keys of this row, and of the block's last
    float q[32], o[32];
    const __nv_bfloat16* qrow = p.q + (int64_t)(start + i) * p.q_stride + (h * p.G + g) * kD + part * 32;
#pragma unroll
    for (int d = 0; d < 32; ++d) {
        q[d] = __bfloat162float(qrow[d]);
        o[d] = 0.f;
    }
    float m = kNegInf, l = 0.f;
    for (int j0 = 0; j0 < most; j0 += kKeys) {
        __syncthreads();
        for (int e = threadIdx.x; e < kKeys * kD; e += kThreads) {
            const int j = j0 + e / kD, d = e % kD;
            float k = 0.f, v = 0.f;
            if (j < most) {
                const int page = __ldcg(p.page_table + (size_t)b * p.max_pages + (j >> p.ps_log2));
                if (page >= 0 && page < p.P) {
                    const size_t at = (((((size_t)page * p.Hkv + h) << p.ps_log2) + (j & ((1 << p.ps_log2) - 1)))) * kD + d;
                    k = __bfloat162float(p.k_pages[at]);
                    v = __bfloat162float(p.v_pages[at]);
                }
            }
            sk[e / kD][d] = k;
            sv[e / kD][d] = v;
        }
        __syncthreads();
        for (int j = 0; j < kKeys; ++j) {
            float s = 0.f;
#pragma unroll
            for (int d = 0; d < 32; ++d) s += q[d] * sk[j][part * 32 + d];
            s += __shfl_xor_sync(0xffffffffu, s, 1);
            s += __shfl_xor_sync(0xffffffffu, s, 2);
            s *= p.scale_log2;
            if (j0 + j >= seen) continue;
            const float m_new = fmaxf(m, s);
            const float keep = exp2f(m - m_new), w = exp2f(s - m_new);
            l = l * keep + w;
            m = m_new;
#pragma unroll
            for (int d = 0; d < 32; ++d) o[d] = o[d] * keep + w * sv[j][part * 32 + d];
        }
    }
    if (!live) return;
    const float inv = l > 0.f ? 1.f / l : 0.f;
    __nv_bfloat16* dst = p.out + ((int64_t)(start + i) * p.Hq + h * p.G + g) * kD + part * 32;
#pragma unroll
    for (int d = 0; d < 32; ++d) dst[d] = __float2bfloat16(o[d] * inv);
}

}  // namespace

size_t chunk_attention_workspace_bytes(const cs_attn_dims&, int, int) { return 256; }

cs_status launch_chunk_attention(const cs_attn_dims& d, const void* q, int64_t q_stride, int tokens,
                                 const void* k_pages, const void* v_pages, const int32_t* page_table,
                                 const int32_t* ctx_lens, const int32_t* q_starts, void* out, void* workspace,
                                 cudaStream_t stream) {
    ChunkParams p{};
    p.batch = RaggedBatch{ctx_lens, q_starts, d.batch, tokens, q_starts ? 0 : tokens / d.batch,
                          d.max_pages_per_seq * d.page_size};
    p.q = static_cast<const __nv_bfloat16*>(q);
    p.k_pages = static_cast<const __nv_bfloat16*>(k_pages);
    p.v_pages = static_cast<const __nv_bfloat16*>(v_pages);
    p.page_table = page_table;
    p.out = static_cast<__nv_bfloat16*>(out);
    p.q_stride = q_stride;
    p.Hq = d.n_q_heads;
    p.Hkv = d.n_kv_heads;
    p.G = d.n_q_heads / d.n_kv_heads;
    while ((1 << p.ps_log2) < d.page_size) ++p.ps_log2;
    p.max_pages = d.max_pages_per_seq;
    p.P = d.num_pages;
    p.scale_log2 = (d.sm_scale > 0.f ? d.sm_scale : 1.0f / sqrtf((float)kD)) * 1.4426950408889634f;
    cudaError_t e = cudaMemsetAsync(workspace, 0, 4, stream);
    if (e != cudaSuccess) return cuda_fail(e, "cudaMemsetAsync");
    const long long blocks = ((long long)tokens * p.G) / kRows + d.batch + 1;
    e = launch_dependent(chunk_attention_kernel, dim3((unsigned)blocks, (unsigned)p.Hkv), dim3(kThreads), 0, stream, p);
    return e == cudaSuccess ? CS_OK : cuda_fail(e, "chunk_attention_kernel launch");
}

}  // namespace cs
