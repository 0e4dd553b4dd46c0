// packed_cache.cu -- rows into and out of a cache held in 4 bits a value
// (cs_packed_kv_append, cs_packed_kv_read; the format is in cachespec.h).
//
// One thread takes one group of 16 dims of a row of K and of V, whose place it
// looks up once: 32 bytes of bf16 on one side, 8 bytes of codes and a scale byte
// on the other, so the eight threads of a row move its 256, 64 and 8 bytes as
// contiguous segments.  Two neighbours bring in (or store) the four 16-byte
// vectors of their groups in order and exchange the middle ones: every access of
// a warp covers whole sectors.
// 16 requests of 2049 rows, 8 KV heads (172 MB in all): append 38.0 us, 4.5 TB/s,
// bound by the instructions of the rounding (a quotient each, in the definition);
// read 40.0 us, 4.3 TB/s, by the chain of loads that leads to a row.  (A thread a
// group of K or of V, its vectors loaded as they lie: 49 and 55.)
#include "cs_internal.h"
#include "packed.cuh"

namespace cs {
namespace {

constexpr int kThreads = 256;
constexpr uint32_t kLarge = 0x5d80;     // bf16 bits of 2^60: groups from there on, and units up to
constexpr float kSmall = 0x1p-60f;      // 2^-60, are divided (no remainder leaves fp32's range between)

// Quotients by a divisor that the host knows, of numbers below 2^31: one high
// product and a shift (Granlund and Montgomery, 1994).
struct Divisor {
    uint32_t d, mul;
    int shift;
    explicit Divisor(uint32_t d_ = 1) : d(d_), mul(0), shift(0) {
        while ((1ull << shift) < d) ++shift;
        if (shift > 0) mul = (uint32_t)(((1ull << (31 + shift)) + d - 1) / d);
    }
    __device__ __forceinline__ uint32_t operator()(uint32_t n) const {
        return shift > 0 ? __umulhi(n, mul) >> (shift - 1) : n;
    }
};

struct PackedSide {
    uint4* rows;               // [B, n, Hkv, 128] bf16: read by the append, written by the read
    uint8_t* codes;            // [P, Hkv, ps, 64]
    uint8_t* scales;           // [P, Hkv, ps, 8]
    const float* head;         // [Hkv] or NULL
};
struct PackedRowsParams {
    PackedSide k, v;
    const int32_t* page_table; // [B, max_pages]
    const int32_t* ctx_lens;   // [B]
    uint32_t rows;             // B * n * Hkv
    Divisor Hkv, n;
    int ps_log2, max_pages, P;
};

// The row and group of a thread.
struct Place {
    uint32_t row;              // (b, i, h)
    int b, i, h, g;
};
__device__ __forceinline__ Place place_of(const PackedRowsParams& p) {
    Place a;
    a.g = threadIdx.x & (kPackGroups - 1);
    a.row = blockIdx.x * (kThreads / kPackGroups) + threadIdx.x / kPackGroups;
    const uint32_t bi = p.Hkv(a.row);
    a.h = (int)(a.row - bi * p.Hkv.d);
    a.b = (int)p.n(bi);
    a.i = (int)(bi - (uint32_t)a.b * p.n.d);
    return a;
}
// The pool row (page, head, slot) that it lies in; -1 for a row before the first
// key or on a page outside the pool.
__device__ __forceinline__ long long slot_of(const PackedRowsParams& p, const Place& a, int L) {
    const int pos = max(0, min(L, p.max_pages << p.ps_log2)) - (int)p.n.d + a.i;
    if (pos < 0) return -1;
    const int page = __ldcg(p.page_table + (size_t)a.b * p.max_pages + (pos >> p.ps_log2));
    if (page < 0 || page >= p.P) return -1;
    return (((long long)page * p.Hkv.d + a.h) << p.ps_log2) + (pos & ((1 << p.ps_log2) - 1));
}

// Of the four vectors of two neighbours' groups, A0 A1 B0 B1, the first has A0 and
// B0 and gets A0 and A1, the second A1 and B1 and gets B0 and B1; and back.
__device__ __forceinline__ void exchange(uint4& x, uint4& y) {
    const bool odd = threadIdx.x & 1;
    const uint4 give = odd ? x : y;
    uint4 got;
    got.x = __shfl_xor_sync(0xffffffffu, give.x, 1);
    got.y = __shfl_xor_sync(0xffffffffu, give.y, 1);
    got.z = __shfl_xor_sync(0xffffffffu, give.z, 1);
    got.w = __shfl_xor_sync(0xffffffffu, give.w, 1);
    (odd ? x : y) = got;
}
// Where a thread's two vectors lie (before the exchange): 16-byte vectors from the first row on.
__device__ __forceinline__ size_t vector_of(const Place& a) {
    return 2 * ((size_t)a.row * kPackGroups + (a.g & ~1)) + (a.g & 1);
}

__device__ __forceinline__ void append_group(const PackedSide& side, const uint4& x0, const uint4& x1, float head,
                                             long long slot, int g) {
    const uint32_t w[8] = {x0.x, x0.y, x0.z, x0.w, x1.x, x1.y, x1.z, x1.w};
    uint32_t top2 = 0;   // the larger magnitudes of the even and odd dims, NaN where one is
#pragma unroll
    for (int j = 0; j < 8; ++j) asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(top2) : "r"(top2), "r"(w[j] & 0x7fff7fffu));
    float top = fmaxf(__uint_as_float(top2 << 16), __uint_as_float(top2 & 0xffff0000u));
    const bool plain = top2 << 16 < kLarge << 16 && top2 < kLarge << 16;   // (bits of magnitudes are in their order)
    float x[16];
#pragma unroll
    for (int j = 0; j < 16; ++j) x[j] = __uint_as_float(j & 1 ? w[j / 2] & 0xffff0000u : w[j / 2] << 16);
    if (!plain) {   // (a NaN is stored as 0)
        top = 0.f;
#pragma unroll
        for (int j = 0; j < 16; ++j) {
            if (x[j] != x[j]) x[j] = 0.f;
            top = fmaxf(top, fabsf(x[j]));
        }
    }
    const uint32_t scale = to_e4m3(fminf(__fdiv_rn(top, __fmul_rn(6.f, head)), 448.f));
    const float unit = __fmul_rn(f16_lo(scales_f16x2(scale)), head);
    if (plain && unit > kSmall) {
        // x / unit correctly rounded from the correctly rounded reciprocal: one
        // step from x * (1 / unit) with the remainder (Markstein, 1990), three
        // operations in place of a division.  (The remainder as q unit - x: with it a
        // quotient of -0 stays one.)
        const float inv = __frcp_rn(unit);
#pragma unroll
        for (int j = 0; j < 16; ++j) {
            const float q = __fmul_rn(x[j], inv);
            x[j] = __fmaf_rn(-__fmaf_rn(q, unit, -x[j]), inv, q);
        }
    } else {
#pragma unroll
        for (int j = 0; j < 16; ++j) x[j] = unit > 0.f ? __fdiv_rn(x[j], unit) : 0.f;
    }
    uint2 c = make_uint2(0, 0);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        c.x |= to_e2m1x2(x[2 * j], x[2 * j + 1]) << (8 * j);
        c.y |= to_e2m1x2(x[8 + 2 * j], x[8 + 2 * j + 1]) << (8 * j);
    }
    *reinterpret_cast<uint2*>(side.codes + (size_t)slot * kPackCodeBytes + g * 8) = c;
    side.scales[(size_t)slot * kPackGroups + g] = (uint8_t)scale;
}

__global__ void __launch_bounds__(kThreads) packed_append_kernel(const PackedRowsParams p) {
    const Place a = place_of(p);
    wait_prior_grid();
    allow_dependent_launch();
    if (a.row >= p.rows) return;   // (a row's eight threads, so neighbours stay together)
    const int L = __ldcg(p.ctx_lens + a.b);
    const size_t at = vector_of(a);
    uint4 k0 = __ldcg(p.k.rows + at), k1 = __ldcg(p.k.rows + at + 2);
    uint4 v0 = __ldcg(p.v.rows + at), v1 = __ldcg(p.v.rows + at + 2);
    const float k_head = p.k.head ? __ldcg(p.k.head + a.h) : 1.f, v_head = p.v.head ? __ldcg(p.v.head + a.h) : 1.f;
    const long long slot = slot_of(p, a, L);
    exchange(k0, k1);
    exchange(v0, v1);
    if (slot < 0) return;
    append_group(p.k, k0, k1, k_head, slot, a.g);
    append_group(p.v, v0, v1, v_head, slot, a.g);
}

// a b rounded to odd: the odd one of its two neighbours in fp32, or itself.  What is
// then rounded to fewer bits is as if rounded once.
__device__ __forceinline__ float mul_to_odd(float a, float b) {
    const float lo = __fmul_rd(a, b), hi = __fmul_ru(a, b);
    return __float_as_uint(lo) & 1u ? lo : hi;
}

// The values of a group's codes, in bf16.
__device__ __forceinline__ void group_values(const uint2& c, uint32_t s, float head, uint4& x, uint4& y) {
    const uint32_t sc = scales_f16x2(s | s << 8);
    const uint32_t v[8] = {codes_f16x2<0>(c.x), codes_f16x2<1>(c.x), codes_f16x2<2>(c.x), codes_f16x2<3>(c.x),
                           codes_f16x2<0>(c.y), codes_f16x2<1>(c.y), codes_f16x2<2>(c.y), codes_f16x2<3>(c.y)};
    uint32_t r[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const uint32_t z = mul_f16x2(v[j], sc);
        r[j] = pack_bf16x2(mul_to_odd(f16_lo(z), head), mul_to_odd(f16_hi(z), head));
    }
    x = make_uint4(r[0], r[1], r[2], r[3]);
    y = make_uint4(r[4], r[5], r[6], r[7]);
}

__global__ void __launch_bounds__(kThreads) packed_read_kernel(const PackedRowsParams p) {
    const Place a = place_of(p);
    wait_prior_grid();
    allow_dependent_launch();
    if (a.row >= p.rows) return;
    const long long slot = slot_of(p, a, __ldcg(p.ctx_lens + a.b));
    uint4 k0 = make_uint4(0, 0, 0, 0), k1 = k0, v0 = k0, v1 = k0;
    if (slot >= 0) {
        const size_t code = (size_t)slot * kPackCodeBytes + a.g * 8, scale = (size_t)slot * kPackGroups + a.g;
        const uint2 kc = __ldcg(reinterpret_cast<const uint2*>(p.k.codes + code));
        const uint2 vc = __ldcg(reinterpret_cast<const uint2*>(p.v.codes + code));
        const uint32_t ks = __ldcg(p.k.scales + scale), vs = __ldcg(p.v.scales + scale);
        const float k_head = p.k.head ? __ldcg(p.k.head + a.h) : 1.f, v_head = p.v.head ? __ldcg(p.v.head + a.h) : 1.f;
        group_values(kc, ks, k_head, k0, k1);
        group_values(vc, vs, v_head, v0, v1);
    }
    const size_t at = vector_of(a);
    exchange(k0, k1);
    p.k.rows[at] = k0;
    p.k.rows[at + 2] = k1;
    exchange(v0, v1);
    p.v.rows[at] = v0;
    p.v.rows[at + 2] = v1;
}

cs_status launch_rows(void (*kern)(const PackedRowsParams), const cs_attn_dims& d, const cs_packed_pool& pool,
                      void* k_rows, void* v_rows, const int32_t* page_table, const int32_t* ctx_lens, int n,
                      const char* what, cudaStream_t stream) {
    const long long rows = (long long)d.batch * n * d.n_kv_heads;
    if ((long long)d.batch * n > 0x7fffffffLL || rows > 0x7fffffffLL)
        return fail(CS_ERR_UNSUPPORTED, "more than 2^31 rows in one call");
    PackedRowsParams p{};
    p.k = PackedSide{static_cast<uint4*>(k_rows), static_cast<uint8_t*>(pool.k_codes), static_cast<uint8_t*>(pool.k_scales),
                     pool.k_head_scale};
    p.v = PackedSide{static_cast<uint4*>(v_rows), static_cast<uint8_t*>(pool.v_codes), static_cast<uint8_t*>(pool.v_scales),
                     pool.v_head_scale};
    p.page_table = page_table;
    p.ctx_lens = ctx_lens;
    p.rows = (uint32_t)rows;
    p.Hkv = Divisor((uint32_t)d.n_kv_heads);
    p.n = Divisor((uint32_t)n);
    while ((1 << p.ps_log2) < d.page_size) ++p.ps_log2;
    p.max_pages = d.max_pages_per_seq;
    p.P = d.num_pages;
    const unsigned blocks = (unsigned)((rows + kThreads / kPackGroups - 1) / (kThreads / kPackGroups));
    const cudaError_t e = launch_dependent(kern, dim3(blocks), dim3(kThreads), 0, stream, p);
    return e == cudaSuccess ? CS_OK : cuda_fail(e, what);
}

}  // namespace

cs_status launch_packed_append(const cs_attn_dims& d, const cs_packed_pool& pool, const void* new_k, const void* new_v,
                               const int32_t* page_table, const int32_t* ctx_lens, int n_new, cudaStream_t stream) {
    return launch_rows(packed_append_kernel, d, pool, const_cast<void*>(new_k), const_cast<void*>(new_v), page_table,
                       ctx_lens, n_new, "packed_append_kernel launch", stream);
}

cs_status launch_packed_read(const cs_attn_dims& d, const cs_packed_pool& pool, const int32_t* page_table,
                             const int32_t* ctx_lens, int n_rows, void* out_k, void* out_v, cudaStream_t stream) {
    return launch_rows(packed_read_kernel, d, pool, out_k, out_v, page_table, ctx_lens, n_rows,
                       "packed_read_kernel launch", stream);
}

}  // namespace cs
