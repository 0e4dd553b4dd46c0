// packed_attention.cu -- verify attention over a cache held in 4 bits a value
// (cs_packed_verify_attention): o = softmax_j(scale q . K_j) V_j with K and V
// the values that the codes stand for (packed.cuh).
//
// One CTA per (request, query head, draft row); its warps take every fourth
// key each, a lane four dims, with a running maximum and sum each, joined in
// shared memory at the end.
#include <math.h>

#include "cs_internal.h"
#include "packed.cuh"

namespace cs {
namespace {

constexpr int kWarps = 4;

struct PackedAttnParams {
    const __nv_bfloat16* q;      // [B, R, Hq, D]
    __nv_bfloat16* out;          // [B, R, Hq, D]
    const uint8_t* k_codes;      // [P, Hkv, ps, 64]
    const uint8_t* k_scales;     // [P, Hkv, ps, 8]
    const uint8_t* v_codes;
    const uint8_t* v_scales;
    const float* k_head;         // [Hkv] or NULL
    const float* v_head;
    const int32_t* page_table;   // [B, max_pages]
    const int32_t* ctx_lens;     // [B]
    int Hq, Hkv, G, R, ps, max_pages, P;
    float scale_log2;            // sm_scale * log2(e)
};

__device__ __forceinline__ void four_dims(const uint8_t* codes, const uint8_t* scales, size_t slot, int lane,
                                          float (&x)[4]) {
    const uint32_t c = __ldcg(reinterpret_cast<const uint16_t*>(codes + slot * kPackCodeBytes) + lane);
    const uint32_t s = __ldcg(scales + slot * kPackGroups + lane / 4);
    const uint32_t sc = scales_f16x2(s | s << 8);
    const uint32_t a = mul_f16x2(codes_f16x2<0>(c), sc), b = mul_f16x2(codes_f16x2<1>(c), sc);
    x[0] = f16_lo(a);
    x[1] = f16_hi(a);
    x[2] = f16_lo(b);
    x[3] = f16_hi(b);
}

__global__ void __launch_bounds__(kWarps * 32) packed_attention_kernel(const PackedAttnParams p) {
    __shared__ float s_o[kWarps][kPackDim];
    __shared__ float s_m[kWarps], s_l[kWarps];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int h = blockIdx.x, i = blockIdx.y, b = blockIdx.z;
    const int hk = h / p.G;
    wait_prior_grid();
    allow_dependent_launch();
    const int L = max(0, min(__ldcg(p.ctx_lens + b), p.max_pages * p.ps));
    const int n_keys = max(0, L - p.R + 1 + i);
    const size_t row = (((size_t)b * p.R + i) * p.Hq + h) * kPackDim + 4 * lane;
    const float c = p.scale_log2 * (p.k_head ? __ldcg(p.k_head + hk) : 1.f);
    float q[4], o[4] = {0.f, 0.f, 0.f, 0.f}, m = kNegInf, l = 0.f;
    for (int d = 0; d < 4; ++d) q[d] = __bfloat162float(p.q[row + d]);
    for (int j = warp; j < n_keys; j += kWarps) {
        const int page = __ldcg(p.page_table + (size_t)b * p.max_pages + j / p.ps);
        const bool in = page >= 0 && page < p.P;
        const size_t slot = in ? ((size_t)page * p.Hkv + hk) * p.ps + j % p.ps : 0;
        float k[4] = {0.f, 0.f, 0.f, 0.f}, v[4] = {0.f, 0.f, 0.f, 0.f};
        if (in) {
            four_dims(p.k_codes, p.k_scales, slot, lane, k);
            four_dims(p.v_codes, p.v_scales, slot, lane, v);
        }
        float s = q[0] * k[0] + q[1] * k[1] + q[2] * k[2] + q[3] * k[3];
        for (int off = 16; off > 0; off >>= 1) s += __shfl_xor_sync(0xffffffffu, s, off);
        s *= c;
        const float mn = fmaxf(m, s), a = ex2(m - mn), w = ex2(s - mn);
        l = l * a + w;
        for (int d = 0; d < 4; ++d) o[d] = o[d] * a + w * v[d];
        m = mn;
    }
    for (int d = 0; d < 4; ++d) s_o[warp][4 * lane + d] = o[d];
    if (lane == 0) {
        s_m[warp] = m;
        s_l[warp] = l;
    }
    __syncthreads();
    if (warp != 0) return;
    float M = kNegInf, sum = 0.f, r[4] = {0.f, 0.f, 0.f, 0.f};
    for (int w = 0; w < kWarps; ++w) M = fmaxf(M, s_m[w]);
    for (int w = 0; w < kWarps && M != kNegInf; ++w) {
        const float a = ex2(s_m[w] - M);
        sum += s_l[w] * a;
        for (int d = 0; d < 4; ++d) r[d] += s_o[w][4 * lane + d] * a;
    }
    const float inv = sum > 0.f ? (p.v_head ? __ldcg(p.v_head + hk) : 1.f) / sum : 0.f;
    *reinterpret_cast<uint2*>(p.out + row) =
        make_uint2(pack_bf16x2(r[0] * inv, r[1] * inv), pack_bf16x2(r[2] * inv, r[3] * inv));
}

}  // namespace

size_t packed_attention_workspace_bytes(const cs_attn_dims&, int, int) { return 256; }

cs_status launch_packed_attention(const cs_attn_dims& d, const void* q, const cs_packed_pool& pool,
                                  const int32_t* page_table, const int32_t* ctx_lens, int rows, void* out,
                                  void*, cudaStream_t stream) {
    PackedAttnParams p{};
    p.q = static_cast<const __nv_bfloat16*>(q);
    p.out = static_cast<__nv_bfloat16*>(out);
    p.k_codes = static_cast<const uint8_t*>(pool.k_codes);
    p.k_scales = static_cast<const uint8_t*>(pool.k_scales);
    p.v_codes = static_cast<const uint8_t*>(pool.v_codes);
    p.v_scales = static_cast<const uint8_t*>(pool.v_scales);
    p.k_head = pool.k_head_scale;
    p.v_head = pool.v_head_scale;
    p.page_table = page_table;
    p.ctx_lens = ctx_lens;
    p.Hq = d.n_q_heads;
    p.Hkv = d.n_kv_heads;
    p.G = d.n_q_heads / d.n_kv_heads;
    p.R = rows;
    p.ps = d.page_size;
    p.max_pages = d.max_pages_per_seq;
    p.P = d.num_pages;
    p.scale_log2 = (d.sm_scale > 0.f ? d.sm_scale : 1.0f / sqrtf((float)d.head_dim)) * 1.4426950408889634f;
    if (d.batch > 65535) return fail(CS_ERR_UNSUPPORTED, "batch %d too large for one call", d.batch);
    const cudaError_t e = launch_dependent(packed_attention_kernel, dim3(d.n_q_heads, rows, d.batch), dim3(kWarps * 32),
                                           0, stream, p);
    return e == cudaSuccess ? CS_OK : cuda_fail(e, "packed_attention_kernel launch");
}

}  // namespace cs
