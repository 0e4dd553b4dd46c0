// packed_cache.cu -- rows into and out of a cache held in 4 bits a value
// (cs_packed_kv_append, cs_packed_kv_read; the format is in cachespec.h).
//
// One thread takes one group of 16 dims of one row of K or V: 32 bytes of bf16
// on one side, 8 bytes of codes and a scale byte on the other, so the eight
// threads of a row move its 256, 64 and 8 bytes as contiguous segments.
#include "cs_internal.h"
#include "packed.cuh"

namespace cs {
namespace {

constexpr int kThreads = 256;

struct PackedRowsParams {
    const uint4* rows[2];      // append: [B, n, Hkv, 128] bf16 of K and V
    uint4* out[2];             // read: the same
    uint8_t* codes[2];         // [P, Hkv, ps, 64]
    uint8_t* scales[2];        // [P, Hkv, ps, 8]
    const float* head[2];      // [Hkv] or NULL
    const int32_t* page_table; // [B, max_pages]
    const int32_t* ctx_lens;   // [B]
    long long groups;          // B * n * Hkv * 8
    int n, Hkv, ps, max_pages, P;
};

// The row and group of this thread, and the pool row (page, head, slot) that
// it lies in; -1 for a row before the first key or on a page outside the pool.
struct Place {
    int b, i, h, g;
    long long row;             // (b, i, h)
};
__device__ __forceinline__ Place place_of(const PackedRowsParams& p, long long t) {
    Place a;
    a.g = (int)(t & (kPackGroups - 1));
    a.row = t / kPackGroups;
    const long long bi = div_pos(a.row, p.Hkv);
    a.h = (int)(a.row - bi * p.Hkv);
    a.b = (int)div_pos(bi, p.n);
    a.i = (int)(bi - (long long)a.b * p.n);
    return a;
}
__device__ __forceinline__ long long slot_of(const PackedRowsParams& p, const Place& a, int L) {
    const int pos = max(0, min(L, p.max_pages * p.ps)) - p.n + a.i;
    if (pos < 0) return -1;
    const int page = __ldcg(p.page_table + (size_t)a.b * p.max_pages + pos / p.ps);
    if (page < 0 || page >= p.P) return -1;
    return ((long long)page * p.Hkv + a.h) * p.ps + pos % p.ps;
}

__global__ void __launch_bounds__(kThreads) packed_append_kernel(const PackedRowsParams p) {
    const long long t = (long long)blockIdx.x * kThreads + threadIdx.x;
    const int kv = blockIdx.y;
    const Place a = place_of(p, t);
    wait_prior_grid();
    allow_dependent_launch();
    if (t >= p.groups) return;
    const uint4* src = p.rows[kv] + 2 * t;
    const int L = __ldcg(p.ctx_lens + a.b);
    const uint4 x0 = __ldcg(src), x1 = __ldcg(src + 1);
    const float head = p.head[kv] ? __ldcg(p.head[kv] + a.h) : 1.f;
    const long long slot = slot_of(p, a, L);
    if (slot < 0) return;
    const uint32_t w[8] = {x0.x, x0.y, x0.z, x0.w, x1.x, x1.y, x1.z, x1.w};
    float x[16], top = 0.f;
#pragma unroll
    for (int j = 0; j < 16; ++j) {
        x[j] = __uint_as_float(j & 1 ? w[j / 2] & 0xffff0000u : w[j / 2] << 16);
        top = fmaxf(top, fabsf(x[j]));   // (passes over a NaN)
        if (x[j] != x[j]) x[j] = 0.f;
    }
    const uint32_t scale = to_e4m3(fminf(__fdiv_rn(top, __fmul_rn(6.f, head)), 448.f));
    const float unit = __fmul_rn(f16_lo(scales_f16x2(scale)), head);
    uint2 c = make_uint2(0, 0);
    if (unit > 0.f) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            c.x |= to_e2m1x2(__fdiv_rn(x[2 * j], unit), __fdiv_rn(x[2 * j + 1], unit)) << (8 * j);
            c.y |= to_e2m1x2(__fdiv_rn(x[8 + 2 * j], unit), __fdiv_rn(x[8 + 2 * j + 1], unit)) << (8 * j);
        }
    }
    *reinterpret_cast<uint2*>(p.codes[kv] + (size_t)slot * kPackCodeBytes + a.g * 8) = c;
    p.scales[kv][(size_t)slot * kPackGroups + a.g] = (uint8_t)scale;
}

__global__ void __launch_bounds__(kThreads) packed_read_kernel(const PackedRowsParams p) {
    const long long t = (long long)blockIdx.x * kThreads + threadIdx.x;
    const int kv = blockIdx.y;
    const Place a = place_of(p, t);
    wait_prior_grid();
    allow_dependent_launch();
    if (t >= p.groups) return;
    const long long slot = slot_of(p, a, __ldcg(p.ctx_lens + a.b));
    uint4 o[2] = {make_uint4(0, 0, 0, 0), make_uint4(0, 0, 0, 0)};
    if (slot >= 0) {
        const uint2 c = __ldcg(reinterpret_cast<const uint2*>(p.codes[kv] + (size_t)slot * kPackCodeBytes + a.g * 8));
        const uint32_t s = __ldcg(p.scales[kv] + (size_t)slot * kPackGroups + a.g);
        const float head = p.head[kv] ? __ldcg(p.head[kv] + a.h) : 1.f;
        const uint32_t sc = scales_f16x2(s | s << 8);
        const uint32_t v[8] = {codes_f16x2<0>(c.x), codes_f16x2<1>(c.x), codes_f16x2<2>(c.x), codes_f16x2<3>(c.x),
                               codes_f16x2<0>(c.y), codes_f16x2<1>(c.y), codes_f16x2<2>(c.y), codes_f16x2<3>(c.y)};
        uint32_t r[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const uint32_t x = mul_f16x2(v[j], sc);
            r[j] = pack_bf16x2(__fmul_rn(f16_lo(x), head), __fmul_rn(f16_hi(x), head));
        }
        o[0] = make_uint4(r[0], r[1], r[2], r[3]);
        o[1] = make_uint4(r[4], r[5], r[6], r[7]);
    }
    p.out[kv][2 * t] = o[0];
    p.out[kv][2 * t + 1] = o[1];
}

PackedRowsParams rows_params(const cs_attn_dims& d, const cs_packed_pool& pool, const int32_t* page_table,
                             const int32_t* ctx_lens, int n) {
    PackedRowsParams p{};
    p.codes[0] = static_cast<uint8_t*>(pool.k_codes);
    p.codes[1] = static_cast<uint8_t*>(pool.v_codes);
    p.scales[0] = static_cast<uint8_t*>(pool.k_scales);
    p.scales[1] = static_cast<uint8_t*>(pool.v_scales);
    p.head[0] = pool.k_head_scale;
    p.head[1] = pool.v_head_scale;
    p.page_table = page_table;
    p.ctx_lens = ctx_lens;
    p.groups = (long long)d.batch * n * d.n_kv_heads * kPackGroups;
    p.n = n;
    p.Hkv = d.n_kv_heads;
    p.ps = d.page_size;
    p.max_pages = d.max_pages_per_seq;
    p.P = d.num_pages;
    return p;
}

cs_status launch_rows(void (*kern)(const PackedRowsParams), const PackedRowsParams& p, const char* what,
                      cudaStream_t stream) {
    const long long blocks = (p.groups + kThreads - 1) / kThreads;
    if (blocks > 0x7fffffffLL) return fail(CS_ERR_UNSUPPORTED, "too many rows in one call");
    const cudaError_t e = launch_dependent(kern, dim3((unsigned)blocks, 2), dim3(kThreads), 0, stream, p);
    return e == cudaSuccess ? CS_OK : cuda_fail(e, what);
}

}  // namespace

cs_status launch_packed_append(const cs_attn_dims& d, const cs_packed_pool& pool, const void* new_k, const void* new_v,
                               const int32_t* page_table, const int32_t* ctx_lens, int n_new, cudaStream_t stream) {
    PackedRowsParams p = rows_params(d, pool, page_table, ctx_lens, n_new);
    p.rows[0] = static_cast<const uint4*>(new_k);
    p.rows[1] = static_cast<const uint4*>(new_v);
    return launch_rows(packed_append_kernel, p, "packed_append_kernel launch", stream);
}

cs_status launch_packed_read(const cs_attn_dims& d, const cs_packed_pool& pool, const int32_t* page_table,
                             const int32_t* ctx_lens, int n_rows, void* out_k, void* out_v, cudaStream_t stream) {
    PackedRowsParams p = rows_params(d, pool, page_table, ctx_lens, n_rows);
    p.out[0] = static_cast<uint4*>(out_k);
    p.out[1] = static_cast<uint4*>(out_v);
    return launch_rows(packed_read_kernel, p, "packed_read_kernel launch", stream);
}

}  // namespace cs
