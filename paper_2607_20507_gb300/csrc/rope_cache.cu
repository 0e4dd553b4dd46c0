// rope_cache.cu -- new tokens' queries and keys turned by their positions, keys and
// values appended to the paged cache in bf16 or in 4 bits (cs_rope_kv_append,
// cs_packed_rope_kv_append; the formulas are in cachespec.h).
//
// A warp takes a token's heads, four at a time: eight threads a row of 128 dims, each
// two 16-byte vectors whose dims pair up with each other (or, of neighbouring pairs and
// of dims that do not turn, with themselves), so that a thread's cosines and sines are
// the same in every head, are read once and multiplied by the norm's weights once.
// Where tokens are few their heads are spread over several warps, as many as make 8 an SM:
// a token's look-ups cost a warp as much as three fours of heads, and so the CTAs of two
// launches fit beside each other (200 tokens of 64 / 8 heads: 4.2 us, 4.6 with 6 and 6.0
// with 12; 400: 5.4, 6.1, 6.7).  Where that leaves a warp more than twelve fours, by the
// fewest rounds of 20 warps an SM times what each takes (1344 tokens of 64 / 8 heads, two
// warps each: 11.4 us, 14.1 with one, 13.7 with three; 2000: 19.3 with one, 20.6 with two,
// 17.7 with three; 4000: 39.6 with one, 36.4 with two).  Two fours are on their way in
// while one is turned, and the first while the token's request, length and page are
// looked up.  28,932 tokens of 64 / 8 heads, normed (1.2 GB in and out): 200-207 us, 5.8 TB/s
// or more, bound by the memory (one four ahead: 208; one CTA a token, its heads in turn: 296).
#include "cs_internal.h"
#include "packed.cuh"
#include "ragged.cuh"

namespace cs {
namespace {

constexpr int kThreads = 128;
constexpr int kRowThreads = 8;                      // threads of a head's row
constexpr int kRows = 32 / kRowThreads;             // heads that a warp takes at once
constexpr int kWarpsPerSm = 8;                      // that tokens are spread over, where they are few
constexpr int kLongShare = 12;                      // fours of a warp that count as many
constexpr int kLookUp = 3;                          // fours that look-ups cost as much as
constexpr int kCtasPerSm = 5;
constexpr float kLarge = 0x1p60f, kSmall = 0x1p-60f;   // between them quotients go without a division

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
    uint32_t q_stride, k_stride, v_stride, q_out_stride;   // (elements)
    float eps;
    int Hq, Hkv, rot, n_positions;
    int ps_log2, max_pages, P;
    int parts;                 // warps of a token
};

// Eight values as four pairs
struct Eight {
    uint64_t v[4];
};
__device__ __forceinline__ Eight unpack8(const uint4& w) {
    const uint32_t u[4] = {w.x, w.y, w.z, w.w};
    Eight x;
#pragma unroll
    for (int j = 0; j < 4; ++j) x.v[j] = f2_pack(__uint_as_float(u[j] << 16), __uint_as_float(u[j] & 0xffff0000u));
    return x;
}
__device__ __forceinline__ uint4 pack8(const Eight& x) {
    uint32_t u[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        float a, b;
        f2_unpack(x.v[j], a, b);
        u[j] = pack_bf16x2(a, b);
    }
    return make_uint4(u[0], u[1], u[2], u[3]);
}
__device__ __forceinline__ uint64_t swapped(uint64_t v) {
    float a, b;
    f2_unpack(v, a, b);
    return f2_pack(b, a);
}

// Half a group (eight dims; the neighbouring thread has the other half) of a row of a
// packed cache, by the rule of cs_packed_kv_append.
__device__ __forceinline__ void store_half_group(const Eight& x0, float head, bool put, uint8_t* codes,
                                                 uint8_t* scales, size_t row, int chunk) {
    float x[8], top = 0.f;
#pragma unroll
    for (int j = 0; j < 4; ++j) f2_unpack(x0.v[j], x[2 * j], x[2 * j + 1]);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        if (x[j] != x[j]) x[j] = 0.f;
        top = fmaxf(top, fabsf(x[j]));
    }
    top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
    const uint32_t scale = to_e4m3(fminf(__fdiv_rn(top, __fmul_rn(6.f, head)), 448.f));
    const float unit = __fmul_rn(f16_lo(scales_f16x2(scale)), head);
    if (top < kLarge && unit > kSmall && unit < kLarge) {
        // x / unit correctly rounded from the correctly rounded reciprocal: one step from
        // x * (1 / unit) with the remainder (Markstein, 1990)
        const float inv = __frcp_rn(unit);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float q = __fmul_rn(x[j], inv);
            x[j] = __fmaf_rn(-__fmaf_rn(q, unit, -x[j]), inv, q);
        }
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = unit > 0.f ? __fdiv_rn(x[j], unit) : 0.f;
    }
    uint32_t c = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) c |= to_e2m1x2(x[2 * j], x[2 * j + 1]) << (8 * j);
    if (!put) return;
    *reinterpret_cast<uint32_t*>(codes + row * kPackCodeBytes + chunk * 4) = c;
    if ((chunk & 1) == 0) scales[row * kPackGroups + chunk / 2] = (uint8_t)scale;
}

// What a thread does to its sixteen dims x and y: x <- x xx + y xy, y <- y yy + x yx (or,
// of neighbouring dims, x <- x xx + x' xy with the pairs of x swapped, and the same of y),
// times 1 / rms where there is a norm.  Dims that do not turn see nothing of their
// partners (0 times an infinity is no 0).
template <bool kNeighbours>
struct Turn {
    Eight xx, xy, yy, yx;
    uint64_t seen;             // of the other dims' bits
    // row: the position's cosines and sines, or NULL for dims that do not turn
    __device__ __forceinline__ Turn(const float* row, int rot, const uint4* norm, int c0, int c1) {
        seen = row ? ~0ull : 0ull;
        // the cosines and sines of pairs 8t .. 8t+7, or (neighbouring dims) of the four of
        // either vector
        float cosv[8], sinv[8], u[8], v[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            cosv[j] = u[j] = v[j] = 1.f;
            sinv[j] = 0.f;
        }
        if (row) {
            const int i0 = kNeighbours ? 4 * c0 : 8 * c0, i1 = kNeighbours ? 4 * c1 : 8 * c0 + 4;
            *reinterpret_cast<float4*>(cosv) = *reinterpret_cast<const float4*>(row + i0);
            *reinterpret_cast<float4*>(cosv + 4) = *reinterpret_cast<const float4*>(row + i1);
            *reinterpret_cast<float4*>(sinv) = *reinterpret_cast<const float4*>(row + rot / 2 + i0);
            *reinterpret_cast<float4*>(sinv + 4) = *reinterpret_cast<const float4*>(row + rot / 2 + i1);
        }
        if (norm) {
            const Eight a = unpack8(norm[c0]), b = unpack8(norm[c1]);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                f2_unpack(a.v[j], u[2 * j], u[2 * j + 1]);
                f2_unpack(b.v[j], v[2 * j], v[2 * j + 1]);
            }
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int i = 2 * j, k = 2 * j + 1;
            if constexpr (kNeighbours) {
                xx.v[j] = f2_pack(u[i] * cosv[j], u[k] * cosv[j]);
                xy.v[j] = f2_pack(u[k] * -sinv[j], u[i] * sinv[j]);
                yy.v[j] = f2_pack(v[i] * cosv[4 + j], v[k] * cosv[4 + j]);
                yx.v[j] = f2_pack(v[k] * -sinv[4 + j], v[i] * sinv[4 + j]);
            } else {
                xx.v[j] = f2_pack(u[i] * cosv[i], u[k] * cosv[k]);
                xy.v[j] = f2_pack(v[i] * -sinv[i], v[k] * -sinv[k]);
                yy.v[j] = f2_pack(v[i] * cosv[i], v[k] * cosv[k]);
                yx.v[j] = f2_pack(u[i] * sinv[i], u[k] * sinv[k]);
            }
            if (!row) xy.v[j] = yx.v[j] = 0x8000000080000000ull;   // -0: what it is added to stays
        }
    }
    __device__ __forceinline__ void operator()(Eight& x, Eight& y, bool norm, float eps) const {
        Eight a, b;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const uint64_t xo = (kNeighbours ? swapped(x.v[j]) : y.v[j]) & seen;
            const uint64_t yo = (kNeighbours ? swapped(y.v[j]) : x.v[j]) & seen;
            a.v[j] = f2_fma(x.v[j], xx.v[j], f2_mul(xo, xy.v[j]));
            b.v[j] = f2_fma(y.v[j], yy.v[j], f2_mul(yo, yx.v[j]));
        }
        if (norm) {   // (the eight threads of the row)
            uint64_t sq = f2_mul(x.v[0], x.v[0]);
#pragma unroll
            for (int j = 1; j < 4; ++j) sq = f2_fma(x.v[j], x.v[j], sq);
#pragma unroll
            for (int j = 0; j < 4; ++j) sq = f2_fma(y.v[j], y.v[j], sq);
            float s0, s1;
            f2_unpack(sq, s0, s1);
            float sum = s0 + s1;
#pragma unroll
            for (int m = 1; m < kRowThreads; m *= 2) sum += __shfl_xor_sync(0xffffffffu, sum, m);
            const float inv = rsqrtf(sum * (1.f / 128) + eps);
            const uint64_t inv2 = f2_pack(inv, inv);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                a.v[j] = f2_mul(a.v[j], inv2);
                b.v[j] = f2_mul(b.v[j], inv2);
            }
        }
        x = a;
        y = b;
    }
};

template <bool kPacked, bool kNeighbours>
__global__ void __launch_bounds__(kThreads, kCtasPerSm) rope_append_kernel(const RopeParams p) {
    const int lane = threadIdx.x & 31, t = lane & (kRowThreads - 1);
    const uint32_t token = blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5);
    const int part = blockIdx.y;
    // the thread's two vectors of a row, and whether they turn
    const int turning = p.rot / 16;     // threads whose vectors do
    const bool turns = t < turning;
    const int c0 = turns ? t : t + turning, c1 = turns ? t + turning : t + 8;
    wait_prior_grid();
    allow_dependent_launch();
    if (token >= (uint32_t)p.batch.tokens) return;

    // fours of heads: those of q, of k, of v; this warp's are part, part + parts, ..
    const int fours_q = (p.Hq + kRows - 1) / kRows, fours_k = (p.Hkv + kRows - 1) / kRows;
    const int fours = fours_q + 2 * fours_k;
    const int sub = lane / kRowThreads;
    // the next four and the one behind it
    uint4 w0 = make_uint4(0, 0, 0, 0), w1 = w0, n0 = w0, n1 = w0;
    auto fetch = [&](int four, uint4& w0, uint4& w1) {
        const bool is_q = four < fours_q, is_v = four >= fours_q + fours_k;
        const int head = (four - (is_q ? 0 : is_v ? fours_q + fours_k : fours_q)) * kRows + sub;
        if (head >= (is_q ? p.Hq : p.Hkv)) return;
        const __nv_bfloat16* from = is_q ? p.q : is_v ? p.v : p.k;
        const uint32_t stride = is_q ? p.q_stride : is_v ? p.v_stride : p.k_stride;
        const uint4* src = reinterpret_cast<const uint4*>(from + (uint64_t)token * stride + (uint32_t)head * 128u);
        w0 = __ldcg(src + c0);
        w1 = __ldcg(src + c1);
    };
    int four = part;
    fetch(four, w0, w1);
    fetch(four + p.parts, n0, n1);
    auto advance = [&](uint4& a, uint4& c) {
        a = w0;
        c = w1;
        w0 = n0;
        w1 = n1;
        fetch(four + 2 * p.parts, n0, n1);
    };
    const int b = p.batch.request_of((int)token, lane);
    if (b < 0) return;
    int start, n, L;
    p.batch.rows_of(b, start, n, L);
    if ((unsigned)((int)token - start) >= (unsigned)n) return;
    const int key = L - n + ((int)token - start);
    const int at = p.positions ? __ldcg(p.positions + token) : key;
    if (at < 0 || at >= p.n_positions) return;
    int page = -1;
    if (key >= 0) page = __ldcg(p.page_table + (size_t)b * p.max_pages + (key >> p.ps_log2));
    const float* const row = turns ? p.cos_sin + (size_t)at * p.rot : nullptr;
    if (four < fours_q) {
        const Turn<kNeighbours> turn(row, p.rot, p.q_norm, c0, c1);
        uint4* const out = reinterpret_cast<uint4*>(p.q_out + (uint64_t)token * p.q_out_stride);
        for (; four < fours_q; four += p.parts) {
            uint4 a, c;
            advance(a, c);
            Eight x = unpack8(a), y = unpack8(c);
            turn(x, y, p.q_norm != nullptr, p.eps);
            const int h = four * kRows + sub;
            if (h < p.Hq) {
                out[h * 16 + c0] = pack8(x);
                out[h * 16 + c1] = pack8(y);
            }
        }
    }
    if (page < 0 || page >= p.P) return;
    const size_t slot0 = (((size_t)page * p.Hkv) << p.ps_log2) + (key & ((1 << p.ps_log2) - 1));   // of head 0
    if (four < fours_q + fours_k) {
        const Turn<kNeighbours> turn(row, p.rot, p.k_norm, c0, c1);
        for (; four < fours_q + fours_k; four += p.parts) {
            uint4 a, c;
            advance(a, c);
            Eight x = unpack8(a), y = unpack8(c);
            turn(x, y, p.k_norm != nullptr, p.eps);
            const int h = (four - fours_q) * kRows + sub;
            const size_t slot = slot0 + ((size_t)h << p.ps_log2);
            if constexpr (kPacked) {
                const bool put = h < p.Hkv;
                const float head = put && p.k_head ? __ldcg(p.k_head + h) : 1.f;
                store_half_group(x, head, put, static_cast<uint8_t*>(p.k_rows), p.k_scales, slot, c0);
                store_half_group(y, head, put, static_cast<uint8_t*>(p.k_rows), p.k_scales, slot, c1);
            } else if (h < p.Hkv) {
                uint4* dst = reinterpret_cast<uint4*>(p.k_rows) + slot * 16;
                dst[c0] = pack8(x);
                dst[c1] = pack8(y);
            }
        }
    }
    for (; four < fours; four += p.parts) {
        uint4 a, c;
        advance(a, c);
        const int h = (four - fours_q - fours_k) * kRows + sub;
        const size_t slot = slot0 + ((size_t)h << p.ps_log2);
        if constexpr (kPacked) {
            const bool put = h < p.Hkv;
            const float head = put && p.v_head ? __ldcg(p.v_head + h) : 1.f;
            const Eight x = unpack8(a), y = unpack8(c);
            store_half_group(x, head, put, static_cast<uint8_t*>(p.v_rows), p.v_scales, slot, c0);
            store_half_group(y, head, put, static_cast<uint8_t*>(p.v_rows), p.v_scales, slot, c1);
        } else if (h < p.Hkv) {
            // (as they are, whatever their bits)
            uint4* dst = reinterpret_cast<uint4*>(p.v_rows) + slot * 16;
            dst[c0] = a;
            dst[c1] = c;
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
    p.q_stride = (uint32_t)r.q_stride;
    p.k_stride = (uint32_t)r.k_stride;
    p.v_stride = (uint32_t)r.v_stride;
    p.q_out_stride = (uint32_t)r.q_out_stride;
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
    // as many warps as there is room for, each a token's share of fours
    const int fours = (p.Hq + kRows - 1) / kRows + 2 * ((p.Hkv + kRows - 1) / kRows);
    const long long sms = current_sm_count(), room = sms * kWarpsPerSm / r.tokens;
    p.parts = room < 1 ? 1 : room < fours ? (int)room : fours;
    auto share = [&](int parts) { return (fours + parts - 1) / parts; };
    if (share(p.parts) > kLongShare) {
        const long long at_once = sms * kCtasPerSm * (kThreads / 32);
        long long best = 0;
        for (int parts = p.parts; share(parts) > kLookUp; ++parts) {
            const long long cost = (r.tokens * (long long)parts + at_once - 1) / at_once * (kLookUp + share(parts));
            if (best == 0 || cost < best) {
                best = cost;
                p.parts = parts;
            }
        }
    }
    const dim3 grid((unsigned)((r.tokens + kThreads / 32 - 1) / (kThreads / 32)), (unsigned)p.parts);
    const cudaError_t e = launch_dependent(kern, grid, dim3(kThreads), 0, stream, p);
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
