// rope_cache.cu -- new tokens' queries and keys turned by their positions, keys and
// values appended to the paged cache in bf16 or in 4 bits (cs_rope_kv_append,
// cs_packed_rope_kv_append; the formulas are in cachespec.h).
//
// A token is one CTA's: eight threads take a head's row of 128 dims, each two 16-byte
// vectors whose dims pair up with each other (or, of neighbouring pairs and of dims
// that do not turn, with themselves), so that a thread's cosines and sines are the
// same in every head and are read once.
#include "cs_internal.h"
#include "packed.cuh"
#include "ragged.cuh"

namespace cs {
namespace {

constexpr int kThreads = 256;
constexpr int kRowThreads = 8;                      // threads of a head's row
constexpr int kRowsAtOnce = kThreads / kRowThreads;

struct RopeParams {
    RaggedBatch batch;
    const __nv_bfloat16 *q, *k, *v;
    const float* cos_sin;      // [n_positions, rot]
    const int32_t* positions;  // [tokens] or NULL
    const uint4 *q_norm, *k_norm;
    __nv_bfloat16* q_out;
    void *k_rows, *v_rows;     // pools: bf16 rows, or codes
    uint8_t *k_scales, *v_scales;
    const float *k_head, *v_head;
    const int32_t* page_table;
    int64_t q_stride, k_stride, v_stride, q_out_stride;
    float eps;
    int Hq, Hkv, rot, n_positions;
    int ps_log2, max_pages, P;
};

__device__ __forceinline__ void unpack8(const uint4& w, float (&x)[8]) {
    const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        x[2 * j] = __uint_as_float(u[j] << 16);
        x[2 * j + 1] = __uint_as_float(u[j] & 0xffff0000u);
    }
}
__device__ __forceinline__ uint4 pack8(const float (&x)[8]) {
    return make_uint4(pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]), pack_bf16x2(x[4], x[5]), pack_bf16x2(x[6], x[7]));
}

// Half a group (eight dims; the neighbouring thread has the other half) of a row of a
// packed cache, by the rule of cs_packed_kv_append.
__device__ __forceinline__ void store_half_group(const float (&x0)[8], float head, uint8_t* codes, uint8_t* scales,
                                                 size_t row, int chunk) {
    float x[8], top = 0.f;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        x[j] = x0[j] != x0[j] ? 0.f : x0[j];
        top = fmaxf(top, fabsf(x[j]));
    }
    top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
    const uint32_t scale = to_e4m3(fminf(__fdiv_rn(top, __fmul_rn(6.f, head)), 448.f));
    const float unit = __fmul_rn(f16_lo(scales_f16x2(scale)), head);
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = unit > 0.f ? __fdiv_rn(x[j], unit) : 0.f;
    uint32_t c = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) c |= to_e2m1x2(x[2 * j], x[2 * j + 1]) << (8 * j);
    if (!codes) return;
    *reinterpret_cast<uint32_t*>(codes + row * kPackCodeBytes + chunk * 4) = c;
    if ((chunk & 1) == 0) scales[row * kPackGroups + chunk / 2] = (uint8_t)scale;
}

template <bool kPacked, bool kNeighbours>
__global__ void __launch_bounds__(kThreads) rope_append_kernel(const RopeParams p) {
    const int t = threadIdx.x & (kRowThreads - 1), lane = threadIdx.x & 31;
    const int64_t token = blockIdx.x;
    // the thread's two vectors of a row, and whether they turn
    const int turning = p.rot / 16;     // threads whose vectors do
    const bool turns = t < turning;
    const int c0 = turns ? t : t + turning, c1 = turns ? t + turning : t + 8;
    wait_prior_grid();
    allow_dependent_launch();
    const int b = p.batch.request_of((int)token, lane);
    if (b < 0) return;
    int start, n, L;
    p.batch.rows_of(b, start, n, L);
    const int key = L - n + ((int)token - start);
    const int at = p.positions ? __ldcg(p.positions + token) : key;
    if (at < 0 || at >= p.n_positions) return;
    int page = -1;
    if (key >= 0) page = __ldcg(p.page_table + (size_t)b * p.max_pages + (key >> p.ps_log2));
    const bool stored = page >= 0 && page < p.P;

    // the cosines and sines of pairs 8t .. 8t+7, or (neighbouring dims) of the four of
    // either vector
    float cosv[8], sinv[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        cosv[j] = 1.f;
        sinv[j] = 0.f;
    }
    if (turns) {
        const float* row = p.cos_sin + (size_t)at * p.rot;
        const int i0 = kNeighbours ? 4 * c0 : 8 * t, i1 = kNeighbours ? 4 * c1 : 8 * t + 4;
        *reinterpret_cast<float4*>(cosv) = *reinterpret_cast<const float4*>(row + i0);
        *reinterpret_cast<float4*>(cosv + 4) = *reinterpret_cast<const float4*>(row + i1);
        row += p.rot / 2;
        *reinterpret_cast<float4*>(sinv) = *reinterpret_cast<const float4*>(row + i0);
        *reinterpret_cast<float4*>(sinv + 4) = *reinterpret_cast<const float4*>(row + i1);
    }
    const int rows = p.Hq + 2 * p.Hkv;
    const int first_row = threadIdx.x / kRowThreads, first_of_warp = first_row & ~3;
    for (int r0 = 0; r0 + first_of_warp < rows; r0 += kRowsAtOnce) {
        const int r = r0 + first_row;
        const bool live = r < rows;
        const bool is_q = r < p.Hq, is_v = r >= p.Hq + p.Hkv;
        const int h = is_q ? r : is_v ? r - p.Hq - p.Hkv : r - p.Hq;
        const __nv_bfloat16* from = is_q ? p.q + token * p.q_stride : is_v ? p.v + token * p.v_stride : p.k + token * p.k_stride;
        uint4 w0 = make_uint4(0, 0, 0, 0), w1 = w0;
        if (live) {
            const uint4* src = reinterpret_cast<const uint4*>(from + h * 128);
            w0 = __ldcg(src + c0);
            w1 = __ldcg(src + c1);
        }
        float x[8], y[8];
        unpack8(w0, x);
        unpack8(w1, y);
        const uint4* norm = is_v ? nullptr : is_q ? p.q_norm : p.k_norm;
        float sum = 0.f;
#pragma unroll
        for (int j = 0; j < 8; ++j) sum += x[j] * x[j] + y[j] * y[j];
#pragma unroll
        for (int m = 1; m < kRowThreads; m *= 2) sum += __shfl_xor_sync(0xffffffffu, sum, m);
        if (norm) {
            const float inv = rsqrtf(sum * (1.f / 128) + p.eps);
            float u[8], v[8];
            unpack8(norm[c0], u);
            unpack8(norm[c1], v);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                x[j] *= inv * u[j];
                y[j] *= inv * v[j];
            }
        }
        if (!is_v && turns) {
            if constexpr (kNeighbours) {
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const float a = x[2 * j], c = x[2 * j + 1], d = y[2 * j], e = y[2 * j + 1];
                    x[2 * j] = a * cosv[j] - c * sinv[j];
                    x[2 * j + 1] = c * cosv[j] + a * sinv[j];
                    y[2 * j] = d * cosv[4 + j] - e * sinv[4 + j];
                    y[2 * j + 1] = e * cosv[4 + j] + d * sinv[4 + j];
                }
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const float a = x[j], c = y[j];
                    x[j] = a * cosv[j] - c * sinv[j];
                    y[j] = c * cosv[j] + a * sinv[j];
                }
            }
        }
        const size_t slot = ((((size_t)(stored ? page : 0) * p.Hkv + h) << p.ps_log2) + (key & ((1 << p.ps_log2) - 1)));
        if (live && is_q) {
            uint4* dst = reinterpret_cast<uint4*>(p.q_out + token * p.q_out_stride + h * 128);
            dst[c0] = pack8(x);
            dst[c1] = pack8(y);
        } else if (!kPacked && live && stored) {
            // (values as they are, whatever their bits)
            uint4* dst = reinterpret_cast<uint4*>(is_v ? p.v_rows : p.k_rows) + slot * 16;
            dst[c0] = is_v ? w0 : pack8(x);
            dst[c1] = is_v ? w1 : pack8(y);
        }
        if constexpr (kPacked) {
            // (a warp has rows of q and of k: neighbours have one row)
            if (__any_sync(0xffffffffu, live && !is_q)) {
                const bool put = live && !is_q && stored;
                const float* heads = is_v ? p.v_head : p.k_head;
                const float head = put && heads ? __ldcg(heads + h) : 1.f;
                uint8_t* codes = put ? static_cast<uint8_t*>(is_v ? p.v_rows : p.k_rows) : nullptr;
                uint8_t* scales = is_v ? p.v_scales : p.k_scales;
                store_half_group(x, head, codes, scales, slot, c0);
                store_half_group(y, head, codes, scales, slot, c1);
            }
        }
    }
}

int log2_of(int x) {
    int s = 0;
    while ((1 << s) < x) ++s;
    return s;
}

cs_status launch(const cs_attn_dims& d, const cs_rope_dims& r, RopeParams& p, bool packed, const int32_t* page_table,
                 const int32_t* ctx_lens, const int32_t* q_starts, cudaStream_t stream) {
    p.batch = RaggedBatch{ctx_lens, q_starts, d.batch, r.tokens, q_starts ? 0 : r.tokens / d.batch,
                          d.max_pages_per_seq * d.page_size};
    p.page_table = page_table;
    p.q_stride = r.q_stride;
    p.k_stride = r.k_stride;
    p.v_stride = r.v_stride;
    p.q_out_stride = r.q_out_stride;
    p.eps = r.norm_eps;
    p.Hq = p.q ? d.n_q_heads : 0;
    p.Hkv = d.n_kv_heads;
    p.rot = r.rot_dim;
    p.n_positions = r.n_positions;
    p.ps_log2 = log2_of(d.page_size);
    p.max_pages = d.max_pages_per_seq;
    p.P = d.num_pages;
    auto kern = packed ? (r.interleaved ? rope_append_kernel<true, true> : rope_append_kernel<true, false>)
                       : (r.interleaved ? rope_append_kernel<false, true> : rope_append_kernel<false, false>);
    const cudaError_t e = launch_dependent(kern, dim3((unsigned)r.tokens), dim3(kThreads), 0, stream, p);
    return e == cudaSuccess ? CS_OK : cuda_fail(e, "rope_append_kernel launch");
}

RopeParams inputs(const void* q, const void* new_k, const void* new_v, const float* cos_sin, const int32_t* positions,
                  const void* q_norm, const void* k_norm, void* q_out) {
    RopeParams p{};
    p.q = static_cast<const __nv_bfloat16*>(q);
    p.k = static_cast<const __nv_bfloat16*>(new_k);
    p.v = static_cast<const __nv_bfloat16*>(new_v);
    p.cos_sin = cos_sin;
    p.positions = positions;
    p.q_norm = static_cast<const uint4*>(q_norm);
    p.k_norm = static_cast<const uint4*>(k_norm);
    p.q_out = static_cast<__nv_bfloat16*>(q_out);
    return p;
}

}  // namespace

cs_status launch_rope_append(const cs_attn_dims& d, const cs_rope_dims& r, const void* q, const void* new_k,
                             const void* new_v, const float* cos_sin, const int32_t* positions, const void* q_norm,
                             const void* k_norm, void* q_out, void* k_pages, void* v_pages, const int32_t* page_table,
                             const int32_t* ctx_lens, const int32_t* q_starts, cudaStream_t stream) {
    RopeParams p = inputs(q, new_k, new_v, cos_sin, positions, q_norm, k_norm, q_out);
    p.k_rows = k_pages;
    p.v_rows = v_pages;
    return launch(d, r, p, false, page_table, ctx_lens, q_starts, stream);
}

cs_status launch_packed_rope_append(const cs_attn_dims& d, const cs_rope_dims& r, const void* q, const void* new_k,
                                    const void* new_v, const float* cos_sin, const int32_t* positions,
                                    const void* q_norm, const void* k_norm, void* q_out, const cs_packed_pool& pool,
                                    const int32_t* page_table, const int32_t* ctx_lens, const int32_t* q_starts,
                                    cudaStream_t stream) {
    RopeParams p = inputs(q, new_k, new_v, cos_sin, positions, q_norm, k_norm, q_out);
    p.k_rows = pool.k_codes;
    p.v_rows = pool.v_codes;
    p.k_scales = static_cast<uint8_t*>(pool.k_scales);
    p.v_scales = static_cast<uint8_t*>(pool.v_scales);
    p.k_head = pool.k_head_scale;
    p.v_head = pool.v_head_scale;
    return launch(d, r, p, true, page_table, ctx_lens, q_starts, stream);
}

}  // namespace cs
