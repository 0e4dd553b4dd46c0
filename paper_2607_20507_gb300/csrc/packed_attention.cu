// packed_attention.cu -- verify attention over a cache held in 4 bits a value
// (cs_packed_verify_attention): o = softmax_j(scale q . K_j) V_j with K and V
// the values that the codes stand for (packed.cuh).
//
// Up to 24 query rows per KV head take the form below, more the tcgen05 form
// (packed_attention_tc.cuh).
//
// Work split.  A span is one (request, KV head) -- with more than 80 query rows
// one of two blocks of them; its keys go in tiles of 128.  The grid holds the
// CTAs that are resident at once, and each takes an equal share of all tiles (a
// span's start counts as `span_x` more).  A span that lies in one CTA is written
// there; one that is cut leaves each piece's normalised output and (maximum,
// sum), which packed_merge_kernel joins.  (A CTA a span would leave the longest
// context to one CTA; pieces of a fixed length would all have to be joined.)
//
// Per CTA: four warps, each with a quarter of a tile's keys and a ring of its
// own in shared memory for them, filled by cp.async (a page piece of 16 keys is
// 1 KB of codes and 128 bytes of scales for K and for V: too little for a bulk
// copy each).  A warp holds all query rows, 8 kNT of them.
//
// Per warp and tile, transposed products on mma.sync (m16n8k16, fp16 operands,
// fp32 sums), so that the padding is to 8 query rows and not to 16:
//   S^T [16 keys x 8 rows] = K Q^T   lane (r, c) = (lane / 4, lane % 4) takes keys
//       r and r + 8 and dims 32 c .. 32 c + 31: 16 bytes of codes a key, which
//       become the eight A fragments in registers.  The dims of a k-step are
//       any 16, the same ones for K and Q, so no code moves between lanes.
//   O^T [16 dims x 8 rows] += V^T P^T  lane (r, c) takes keys 2c, 2c+1, 2c+8, 2c+9
//       and dims 16 r .. 16 r + 15, one scale group: 8 bytes of codes and one
//       scale a key.  The codes of two keys are paired by nibbles (two shifts
//       and two selections for 16 codes) before they become fp16 pairs.
// P^T is S^T's accumulator after movmatrix.  Codes become fp16 by one
// conversion a pair and one product with their scale, both exact.
//
// The running maximum of a row grows only when a score passes it by 2^3 (then
// the sums are rescaled): P = 2^(s - m + 12) lies between 2^-14 and 2^15, where
// fp16 has 11 bits, for weights down to 2^-26 of the largest.  A tile with
// smaller ones takes another turn for them (faint, below): an output may rest
// on them where the codes of the heavier keys are 0.
//
// What bounds it: turning codes into fp16 pairs and these into scaled ones, an
// instruction each on pipes of 64 lanes a clock, with the address and selection
// work around them, and the latencies that 16 warps an SM leave in the open (issue 60%
// busy, ALU 53%: neither at its limit), not the memory: 256 requests of 1024 to 8192
// keys, 4 rows, 8 KV heads, 276 us for 1.37 GB, 4.9 TB/s (the bytes alone take 200).
// 64 requests of 4096 keys: 4 rows 71 us, 8 72, 12 96, 16 98, 20 125, 24 128 (their
// bytes take 44): one row tile more costs its own products and accumulators, so fewer
// CTAs an SM (four, three and two at 128, 168 and 255 registers).
// These are scores that lie within some 2^26 of their row's largest weight.  Each
// turn for faint weights decodes the values again: with scores of 3, 5 and 8 nats'
// deviation 4 rows take 103, 114 and 147 us and 20 rows 234, 286 and 396; with one key 20, 40
// and 60 nats above the rest 108, 124 and 142, and 250, 318 and 392.
#include <limits.h>
#include <math.h>

#include <type_traits>

#include "bounded_wait.cuh"
#include "cs_internal.h"
#include "packed.cuh"

namespace cs {
namespace {

constexpr int kSub = 32;                            // keys of a warp's tile
constexpr int kHalves = kSub / 16;                  // MMA tiles of 16 keys in it
constexpr int kStages = 2;
constexpr int kCodes = kSub * kPackCodeBytes;       // 2048 bytes of codes of K or V
constexpr int kScales = kSub * kPackGroups;         // 256 bytes of scales
constexpr int kStageBytes = 2 * (kCodes + kScales);
constexpr int kMaxBatchPerLaunch = 1024;            // requests whose schedule one launch holds
constexpr int kMaxGrid = 1024;                      // CTAs of a launch at most
constexpr float kPUp = 12.f;                        // P = 2^(s - m + kPUp)
constexpr float kPMax = 15.f;                       // the maximum follows a score that passes 2^kPMax
constexpr float kPMin = -14.f;                      // weights below 2^kPMin are faint: less than 11 bits in fp16
constexpr float kPGone = -126.f;                    // and those below 2^kPGone count as 0

struct Job {             // a cut span that starts in a CTA: its pieces lie in slot0 and the first slots of the CTAs after it
    int b, h, slot0, n;
};

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
    float* part_o;               // [2 grid, n_rows, D] a CTA's first and last piece
    float2* part_ml;             // [2 grid, n_rows] (maximum in log2 units, sum)
    Job* jobs;                   // [grid]
    int* status;                 // device status word
    int Hq, Hkv, G, R, ps, ps_log2, max_pages, P;
    int n_rows, n_all;           // query rows of a span, and of a KV head
    int n_rb, n_spans;           // row blocks of a KV head, spans of a request (Hkv n_rb)
    int b_base, n_batch, span_x;
    float scale_log2;            // sm_scale * log2(e)
};

// warps that share a tile's keys by query rows, and what follows from the count
template <int kNT>
struct Form {
    static constexpr int kWarps = 4;
    static constexpr int kThreads = kWarps * 32;
    static constexpr int kTile = kWarps * kSub;
    static constexpr int kRows = kNT * 8;
    static constexpr int kMinBlocks = kNT == 1 ? 4 : kNT == 2 ? 3 : 2;
    static constexpr int kRing = kWarps * kStages * kStageBytes;
    static constexpr int kQ = kRows * kPackDim * 2;
    static constexpr int kFold = kWarps / 2 * (kRows * kPackDim * 4 + kNT * 32 * 16);
    static constexpr int kSmem = kRing + kQ + kFold + kRows * 8 + kMaxBatchPerLaunch * 4;
    static_assert(kRing >= (kMaxBatchPerLaunch + 1) * 8, "the prefix lies in the ring at the start");
};

struct Cursor {
    int b, h, t, T;
};

__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src, bool in) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(in ? 16 : 0) : "memory");
}
__device__ __forceinline__ void cp_async8(uint32_t dst, const void* src, bool in) {
    asm volatile("cp.async.ca.shared.global [%0], [%1], 8, %2;" ::"r"(dst), "l"(src), "r"(in ? 8 : 0) : "memory");
}
__device__ __forceinline__ void cp_async4(uint32_t dst, const void* src, bool in) {
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(dst), "l"(src), "r"(in ? 4 : 0) : "memory");
}
__device__ __forceinline__ void cp_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int kLeft>
__device__ __forceinline__ void cp_async_wait() {
    asm volatile("cp.async.wait_group %0;" ::"n"(kLeft) : "memory");
}

__device__ __forceinline__ void mma_f16_16816(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, "
        "{%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// an 8 x 8 matrix of 16-bit values over the warp, transposed
__device__ __forceinline__ uint32_t transpose_8x8(uint32_t x) {
    uint32_t r;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(x));
    return r;
}
__device__ __forceinline__ uint32_t pack_f16x2(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
// the low four bits of every byte from a, the high four from b
__device__ __forceinline__ uint32_t nibbles(uint32_t a, uint32_t b) { return (a & 0x0f0f0f0fu) | (b & 0xf0f0f0f0u); }

// Byte offset of 16-byte part `part` of a key's V codes: with the rows and the
// parts exchanged by the key's bits, the eight-byte loads of a half warp (keys
// 0, 2, 4, 6 and one half of the dims) meet every bank once.
__device__ __forceinline__ int v_at(int key, int part) {
    return (key ^ (key >> 2 & 1)) * kPackCodeBytes + (part ^ (key & 2)) * 16;
}

// Tiles of a request of L keys, its spans' units before request b (prefix) and
// the position of unit v.
struct Share {
    Cursor first;
    int n_tiles;
};
__device__ __forceinline__ int tiles_of(int L, int tile) { return max(1, (L + tile - 1) / tile); }

// The first unit of CTA c of G.
__device__ __forceinline__ long long first_unit(int c, long long U, int G) { return div_pos((long long)c * U, G); }
// The CTA that holds unit v.
__device__ __forceinline__ int owner_of(long long v, long long U, int G) {
    return (int)div_pos((v + 1) * G + U - 1, U) - 1;
}

// The share of CTA c of G, by one warp: even lanes place its first unit, odd
// ones the unit past its last (lanes compare 32 requests' starts at a time).
__device__ __forceinline__ Share share_of(int c, long long U, int G, const long long* prefix, const int* lens, int nb,
                                          int n_spans, int X, int tile) {
    const int lane = threadIdx.x & 31;
    const long long v = first_unit(c + (lane & 1), U, G);
    Cursor cur{};
#pragma unroll
    for (int e = 0; e < 2; ++e) {
        const long long ve = __shfl_sync(0xffffffffu, v, e);
        const int far = lane * 32;
        const int blk = nb > 32 ? 31 - __clz(__ballot_sync(0xffffffffu, far < nb && prefix[far] <= ve)) : 0;
        const int b = blk * 32 + lane;
        const int at = blk * 32 + 31 - __clz(__ballot_sync(0xffffffffu, b < nb && prefix[b] <= ve));
        if ((lane & 1) == e) cur.b = at;
    }
    cur.T = tiles_of(lens[cur.b], tile);
    const long long local = v - prefix[cur.b];
    cur.h = (int)div_pos(local, cur.T + X);     // n_spans: past the last unit
    const int in = (int)(local - (long long)cur.h * (cur.T + X));
    cur.t = in > X ? in - X : 0;
    const long long before = prefix[cur.b] - (long long)X * n_spans * cur.b + (long long)cur.h * cur.T + cur.t;
    Share s;
    s.n_tiles = (int)(__shfl_sync(0xffffffffu, before, 1) - __shfl_sync(0xffffffffu, before, 0));
    s.first.b = __shfl_sync(0xffffffffu, cur.b, 0);
    s.first.h = __shfl_sync(0xffffffffu, cur.h, 0);
    s.first.t = __shfl_sync(0xffffffffu, cur.t, 0);
    s.first.T = __shfl_sync(0xffffffffu, cur.T, 0);
    return s;
}

__device__ __forceinline__ void advance(Cursor& c, const int* lens, int nb, int n_spans, int tile) {
    if (++c.t < c.T) return;
    c.t = 0;
    if (++c.h < n_spans) return;
    c.h = 0;
    if (++c.b < nb) c.T = tiles_of(lens[c.b], tile);
}

// The requests' clamped lengths and their spans' tiles before each, into shared
// memory (ends with a block barrier); all tiles.
template <int kThreads>
__device__ __forceinline__ long long build_prefix(const PackedAttnParams& p, int tile, int* lens, long long* prefix,
                                                  long long* wsum) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    long long carry = 0;
    for (int base = 0; base < p.n_batch; base += kThreads) {
        const int b = base + threadIdx.x;
        long long v = 0;
        if (b < p.n_batch) {
            const int L = max(0, min(__ldcg(p.ctx_lens + p.b_base + b), p.max_pages * p.ps));
            lens[b] = L;
            v = (long long)tiles_of(L, tile) * p.n_spans;
        }
        long long inc = v;
#pragma unroll
        for (int off = 1; off < 32; off <<= 1) {
            const long long y = __shfl_up_sync(0xffffffffu, inc, off);
            if (lane >= off) inc += y;
        }
        if (lane == 31) wsum[warp] = inc;
        __syncthreads();
        long long before = carry, all = 0;
        for (int w = 0; w < kThreads / 32; ++w) {
            if (w < warp) before += wsum[w];
            all += wsum[w];
        }
        if (b < p.n_batch) prefix[b] = before + inc - v;
        carry += all;
        __syncthreads();
    }
    return carry;
}

// Four of a query row's dims (a lane's, of the warp that has the row) as fp16,
// brought below 2^15 by a power of two that the whole row shares; back: its inverse.
__device__ __forceinline__ uint2 query_f16(uint2 x, float& back) {
    const float f[4] = {__uint_as_float(x.x << 16), __uint_as_float(x.x & 0xffff0000u), __uint_as_float(x.y << 16),
                        __uint_as_float(x.y & 0xffff0000u)};
    // (of magnitudes, whose order is that of their bits)
    const float top = __uint_as_float(__reduce_max_sync(
        0xffffffffu, __float_as_uint(fmaxf(fmaxf(fabsf(f[0]), fabsf(f[1])), fmaxf(fabsf(f[2]), fabsf(f[3]))))));
    // top = 1.m x 2^e -> 1.m x 2^14; 2^(14 - e) in two halves, neither of which leaves fp32
    const int e = (int)(__float_as_uint(top) >> 23) - 127;
    const int up = top > 0.f ? 14 - e : 0, u0 = up / 2, u1 = up - u0;
    const float s0 = __uint_as_float((uint32_t)(127 + u0) << 23), s1 = __uint_as_float((uint32_t)(127 + u1) << 23);
    back = __uint_as_float((uint32_t)(127 - u0) << 23) * __uint_as_float((uint32_t)(127 - u1) << 23);
    return make_uint2(pack_f16x2(f[0] * s0 * s1, f[1] * s0 * s1), pack_f16x2(f[2] * s0 * s1, f[3] * s0 * s1));
}

template <int kNT>
__global__ void __launch_bounds__(Form<kNT>::kThreads, Form<kNT>::kMinBlocks)
packed_attention_kernel(const PackedAttnParams p) {
    using F = Form<kNT>;
    extern __shared__ uint4 smem_raw[];
    uint8_t* smem = reinterpret_cast<uint8_t*>(smem_raw);
    uint4* s_q = reinterpret_cast<uint4*>(smem + F::kRing);                       // [row tile][4][lane] B fragments
    float4* s_fold = reinterpret_cast<float4*>(smem + F::kRing + F::kQ);
    float* s_scale = reinterpret_cast<float*>(smem + F::kRing + F::kQ + F::kFold);   // [row] of the scores
    int* s_draft = reinterpret_cast<int*>(s_scale + F::kRows);                    // [row] draft position
    int* s_len = s_draft + F::kRows;
    long long* s_prefix = reinterpret_cast<long long*>(smem);
    __shared__ long long s_wsum[F::kThreads / 32];

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int r = lane >> 2, c = lane & 3;
    const int nb = p.n_batch, X0 = p.span_x;
    // (read from the first span on, after the barriers below)
    for (int row = threadIdx.x; row < F::kRows; row += F::kThreads) s_draft[row] = row / p.G;
    wait_prior_grid();
    allow_dependent_launch();

    const long long W = build_prefix<F::kThreads>(p, F::kTile, s_len, s_prefix, s_wsum);
    // few tiles: one a CTA; else a span's start counts as X tiles
    const int grid = gridDim.x, cta = blockIdx.x;
    const bool few = W <= grid;
    const int X = few ? 0 : X0, Gc = few ? (int)W : grid;
    if (threadIdx.x == 0) {
        p.jobs[cta].n = 0;
        if (cta == 0 && p.b_base == 0) *p.status = 0;
    }
    if (cta >= Gc) return;
    if (X > 0) {
        for (int b = threadIdx.x; b < nb; b += F::kThreads) s_prefix[b] += (long long)X * p.n_spans * b;
        __syncthreads();
    }
    const long long U = W + (long long)X * p.n_spans * nb;
    const Share share = share_of(cta, U, Gc, s_prefix, s_len, nb, p.n_spans, X, F::kTile);
    const int n_tiles = share.n_tiles;
    __syncthreads();   // the prefix gives way to the ring
    if (n_tiles <= 0) return;

    // ---- the ring.  Lane g (mod 4) looks up the page of keys 8 g .. 8 g + 7 of
    // the next tile to load, one tile ahead.
    uint8_t* ring = smem + warp * (kStages * kStageBytes);
    const uint32_t ring_a = smem_u32(ring);
    const int page_rows = p.Hkv * p.ps;
    Cursor cn = share.first;
    int left = n_tiles, stage_in = 0;                 // tiles not looked up yet, the stage that is filled next
    int next_page = -1, next_row = 0;                 // the page of this lane's group, and the row of its keys on it
    bool pending = false;                             // whether a tile is looked up
    auto look_up = [&]() {
        pending = left > 0;
        if (!pending) return;
        --left;
        const int key = cn.t * F::kTile + warp * kSub + 8 * c;
        next_page = -1;
        next_row = cn.h * p.ps + (key & (p.ps - 1));
        if (key < s_len[cn.b])
            next_page = __ldcg(p.page_table + (size_t)(p.b_base + cn.b) * p.max_pages + (key >> p.ps_log2));
        advance(cn, s_len, nb, p.n_spans, F::kTile);
    };
    const uint8_t* k_lane = p.k_codes + r * kPackCodeBytes + c * 16;
    const uint8_t* v_lane = p.v_codes + r * kPackCodeBytes + c * 16;
    const uint8_t* s_lane = (lane < 16 ? p.k_scales : p.v_scales) + c * 16;
    const uint32_t k_to = ring_a + r * kPackCodeBytes + c * 16, v_to = ring_a + kCodes + v_at(r, c);
    const uint32_t s_to = ring_a + 2 * kCodes + lane * 16;
    auto issue = [&]() {
        if (pending) {
            const bool in = next_page >= 0 && next_page < p.P;
            const int row = in ? next_page * page_rows + next_row : -1;
            const uint32_t st = stage_in * kStageBytes;
            look_up();
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const int rw = __shfl_sync(0xffffffffu, row, g);
                const size_t at = (size_t)max(rw, 0) * kPackCodeBytes;
                cp_async16(k_to + st + g * 8 * kPackCodeBytes, k_lane + at, rw >= 0);
                cp_async16(v_to + st + g * 8 * kPackCodeBytes, v_lane + at, rw >= 0);
            }
            const int rw = __shfl_sync(0xffffffffu, row, lane >> 2 & 3);
            cp_async16(s_to + st, s_lane + (size_t)max(rw, 0) * kPackGroups, rw >= 0);
        }
        stage_in = stage_in + 1 == kStages ? 0 : stage_in + 1;
        cp_async_commit();
    };
    look_up();
    for (int i = 0; i < kStages - 1; ++i) issue();
    int stage = 0;

    // ---- spans
    Cursor cur = share.first;
    int done = 0;
    bool first_piece = true;
    while (done < n_tiles) {
        const int n = min(cur.T - cur.t, n_tiles - done);
        const int bg = p.b_base + cur.b, L = s_len[cur.b];
        // the query rows in fp16, brought below 2^15 by a power of two each
        for (int row = warp; row < F::kRows; row += F::kThreads / 32) {
            uint2 x = make_uint2(0, 0);
            if (row < p.n_rows) {
                const int i = s_draft[row];
                const uint32_t* src = reinterpret_cast<const uint32_t*>(
                    p.q + (((size_t)bg * p.R + i) * p.Hq + (size_t)cur.h * p.G + (row - i * p.G)) * kPackDim + 4 * lane);
                x.x = __ldcg(src);
                x.y = __ldcg(src + 1);
            }
            float back;
            const uint2 y = query_f16(x, back);
            uint4* at = s_q + ((row >> 3) * 4 + ((lane & 7) >> 1)) * 32 + (row & 7) * 4 + (lane >> 3);
            reinterpret_cast<uint2*>(at)[lane & 1] = y;
            if (lane == 0) s_scale[row] = p.scale_log2 * back * (p.k_head ? __ldcg(p.k_head + cur.h) : 1.f);
        }
        __syncthreads();

        float o[kNT][8][4], m[kNT][2], l[kNT][2], sc_f[kNT][2];
#pragma unroll
        for (int nt = 0; nt < kNT; ++nt) {
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                m[nt][e] = kNegInf;
                l[nt][e] = 0.f;
                sc_f[nt][e] = s_scale[nt * 8 + 2 * c + e];
            }
#pragma unroll
            for (int i = 0; i < 8; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e) o[nt][i][e] = 0.f;
        }
        const uint4* q_frag = s_q + lane;
        uint4 q_kept[4];   // one row tile's fragments stay in registers
        if constexpr (kNT == 1)
#pragma unroll
            for (int i = 0; i < 4; ++i) q_kept[i] = q_frag[i * 32];

        for (int t = 0; t < n; ++t) {
            cp_async_wait<kStages - 2>();
            __syncwarp();
            const uint8_t* st = ring + stage * kStageBytes;
            stage = stage + 1 == kStages ? 0 : stage + 1;
            issue();   // into the stage that the warp has left
            const int key0 = (cur.t + t) * F::kTile + warp * kSub;
            if (key0 >= L) continue;

            // ---- S^T = K Q^T
            float s[kHalves][kNT][4];
#pragma unroll
            for (int hf = 0; hf < kHalves; ++hf) {
#pragma unroll
                for (int nt = 0; nt < kNT; ++nt)
#pragma unroll
                    for (int e = 0; e < 4; ++e) s[hf][nt][e] = 0.f;
                const uint8_t* kc = st + (16 * hf + r) * kPackCodeBytes + c * 16;
                const uint4 k0 = *reinterpret_cast<const uint4*>(kc);
                const uint4 k1 = *reinterpret_cast<const uint4*>(kc + 8 * kPackCodeBytes);
                const uint8_t* ks = st + 2 * kCodes + (16 * hf + r) * kPackGroups + 2 * c;
                const uint32_t f0 = scales_f16x2(*reinterpret_cast<const uint16_t*>(ks));
                const uint32_t f1 = scales_f16x2(*reinterpret_cast<const uint16_t*>(ks + 8 * kPackGroups));
                const uint32_t w0[4] = {k0.x, k0.y, k0.z, k0.w}, w1[4] = {k1.x, k1.y, k1.z, k1.w};
#pragma unroll
                for (int i = 0; i < 4; ++i) {   // k-steps 2i, 2i + 1: dims 32 c + 8 i ...
                    const uint32_t g0 = __byte_perm(f0, 0, i < 2 ? 0x1010 : 0x3232);
                    const uint32_t g1 = __byte_perm(f1, 0, i < 2 ? 0x1010 : 0x3232);
                    const uint32_t a[2][4] = {
                        {mul_f16x2(codes_f16x2<0>(w0[i]), g0), mul_f16x2(codes_f16x2<0>(w1[i]), g1),
                         mul_f16x2(codes_f16x2<1>(w0[i]), g0), mul_f16x2(codes_f16x2<1>(w1[i]), g1)},
                        {mul_f16x2(codes_f16x2<2>(w0[i]), g0), mul_f16x2(codes_f16x2<2>(w1[i]), g1),
                         mul_f16x2(codes_f16x2<3>(w0[i]), g0), mul_f16x2(codes_f16x2<3>(w1[i]), g1)}};
#pragma unroll
                    for (int nt = 0; nt < kNT; ++nt) {
                        const uint4 qb = kNT == 1 ? q_kept[i] : q_frag[(nt * 4 + i) * 32];
                        mma_f16_16816(s[hf][nt], a[0], qb.x, qb.y);
                        mma_f16_16816(s[hf][nt], a[1], qb.z, qb.w);
                    }
                }
            }
            // ---- x = s - m + 12; lane (r, c): keys r, r + 8 of rows 2c, 2c + 1.
            // Most tiles need no more than that; the others (a key that a row
            // does not see, a maximum that grows, faint weights) branch off here
            // and leave x in s (ready)
            float top = -1.f, low = 0.f;
#pragma unroll
            for (int nt = 0; nt < kNT; ++nt)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    static_assert(kHalves == 2, "");
                    const float up = kPUp - m[nt][e & 1];
                    const float v0 = fmaf(s[0][nt][e], sc_f[nt][e & 1], up), v1 = fmaf(s[1][nt][e], sc_f[nt][e & 1], up);
                    top = fmax3(top, v0, v1);
                    low = fmin3(low, v0, v1);
                }
            const bool edge = key0 + kSub > L - p.R + 1;   // some row does not see some key
            const bool ready = __any_sync(0xffffffffu, top > kPMax || low < kPMin || edge);
            if (ready) {
                low = 0.f;
#pragma unroll
                for (int nt = 0; nt < kNT; ++nt)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const int row = nt * 8 + 2 * c + e;
                        const int last = !edge ? INT_MAX : row < p.n_rows ? L - p.R + s_draft[row] : L - 1;
                        float now = kNegInf;
#pragma unroll
                        for (int hf = 0; hf < kHalves; ++hf)
#pragma unroll
                            for (int k = e; k < 4; k += 2) {
                                const bool seen = key0 + 16 * hf + r + (k & 2) * 4 <= last;
                                s[hf][nt][k] = seen ? s[hf][nt][k] * sc_f[nt][e] : kNegInf;
                                now = fmaxf(now, s[hf][nt][k]);
                            }
#pragma unroll
                        for (int off = 4; off < 32; off <<= 1) now = fmaxf(now, __shfl_xor_sync(0xffffffffu, now, off));
                        if (now - m[nt][e] > kPMax - kPUp) {   // (true for a row's first key: m is -inf)
                            const float a = ex2(m[nt][e] - now);
                            m[nt][e] = now;
                            l[nt][e] *= a;
#pragma unroll
                            for (int i = 0; i < 8; ++i) {
                                o[nt][i][e] *= a;
                                o[nt][i][e + 2] *= a;
                            }
                        }
                        // (a row that has seen no key yet: every score is -inf)
                        const float up = m[nt][e] == kNegInf ? 0.f : kPUp - m[nt][e];
#pragma unroll
                        for (int hf = 0; hf < kHalves; ++hf)
#pragma unroll
                            for (int k = e; k < 4; k += 2) {
                                s[hf][nt][k] += up;
                                if (s[hf][nt][k] > kPGone) low = fminf(low, s[hf][nt][k]);
                            }
                    }
            }
            // f(i, a): the A fragment of V^T for dims 16 r + 2i (rows r) and 16 r + 2i + 1 (rows r + 8)
            auto with_values = [&](int hf, auto f) {
                const uint8_t* vc = st + kCodes + hf * 16 * kPackCodeBytes + 8 * (r & 1);
                const int kv = key0 + 16 * hf;
                const uint2 v0 = *reinterpret_cast<const uint2*>(vc + v_at(2 * c, r >> 1));
                const uint2 v1 = *reinterpret_cast<const uint2*>(vc + v_at(2 * c + 1, r >> 1));
                const uint2 v2 = *reinterpret_cast<const uint2*>(vc + v_at(2 * c + 8, r >> 1));
                const uint2 v3 = *reinterpret_cast<const uint2*>(vc + v_at(2 * c + 9, r >> 1));
                const uint8_t* vs = st + 2 * kCodes + kScales + (16 * hf + 2 * c) * kPackGroups + r;
                uint32_t b0 = vs[0], b1 = vs[kPackGroups], b2 = vs[8 * kPackGroups], b3 = vs[9 * kPackGroups];
                if (kv + 16 > L) {   // slots past the context hold anything
                    if (kv + 2 * c >= L) b0 = 0;
                    if (kv + 2 * c + 1 >= L) b1 = 0;
                    if (kv + 2 * c + 8 >= L) b2 = 0;
                    if (kv + 2 * c + 9 >= L) b3 = 0;
                }
                const uint32_t f01 = scales_f16x2(b0 | b1 << 8), f23 = scales_f16x2(b2 | b3 << 8);
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    const uint32_t w0 = half ? v0.y : v0.x, w1 = half ? v1.y : v1.x;
                    const uint32_t w2 = half ? v2.y : v2.x, w3 = half ? v3.y : v3.x;
                    const uint32_t e01 = nibbles(w0, w1 << 4), o01 = nibbles(w0 >> 4, w1);   // even and odd dims
                    const uint32_t e23 = nibbles(w2, w3 << 4), o23 = nibbles(w2 >> 4, w3);
                    auto dims = [&](auto byte) {
                        constexpr int kByte = decltype(byte)::value;
                        const uint32_t a[4] = {mul_f16x2(codes_f16x2<kByte>(e01), f01), mul_f16x2(codes_f16x2<kByte>(o01), f01),
                                               mul_f16x2(codes_f16x2<kByte>(e23), f23), mul_f16x2(codes_f16x2<kByte>(o23), f23)};
                        f(half * 4 + kByte, a);
                    };
                    dims(std::integral_constant<int, 0>{});
                    dims(std::integral_constant<int, 1>{});
                    dims(std::integral_constant<int, 2>{});
                    dims(std::integral_constant<int, 3>{});
                }
            };
            // faint weights, 28 powers of two at a time, each turn's product scaled back in fp32
            if (ready && __any_sync(0xffffffffu, low < kPMin)) {
                auto is_faint = [&](float v) { return v < kPMin && v > kPGone; };
#pragma unroll
                for (int hf = 0; hf < kHalves; ++hf) {
                    bool faint = false;
#pragma unroll
                    for (int nt = 0; nt < kNT; ++nt)
#pragma unroll
                        for (int e = 0; e < 4; ++e) faint |= is_faint(s[hf][nt][e]);
#pragma unroll 1
                    for (float up = 28.f; __any_sync(0xffffffffu, faint); up += 28.f) {
                        uint32_t pf[kNT][2];
                        faint = false;
#pragma unroll
                        for (int nt = 0; nt < kNT; ++nt) {
                            float w[4];
#pragma unroll
                            for (int e = 0; e < 4; ++e) {
                                float& v = s[hf][nt][e];
                                const bool now = v < kPMin && v + up >= kPMin;
                                w[e] = now ? ex2(v + up) : 0.f;
                                if (now) {
                                    l[nt][e & 1] += ex2(v);
                                    v = kNegInf;
                                }
                                faint |= is_faint(v);
                            }
                            pf[nt][0] = transpose_8x8(pack_f16x2(w[0], w[1]));
                            pf[nt][1] = transpose_8x8(pack_f16x2(w[2], w[3]));
                        }
                        const float down = ex2(-up);
                        with_values(hf, [&](int i, const uint32_t (&a)[4]) {
#pragma unroll
                            for (int nt = 0; nt < kNT; ++nt) {
                                float d[4] = {0.f, 0.f, 0.f, 0.f};
                                mma_f16_16816(d, a, pf[nt][0], pf[nt][1]);
#pragma unroll
                                for (int e = 0; e < 4; ++e) o[nt][i][e] = fmaf(d[e], down, o[nt][i][e]);
                            }
                        });
                    }
                }
            }
            // ---- P = 2^x and O^T += V^T P^T
#pragma unroll
            for (int hf = 0; hf < kHalves; ++hf) {
                uint32_t pb[kNT][2];
#pragma unroll
                for (int nt = 0; nt < kNT; ++nt) {
                    float w[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        w[e] = ex2(fmaf(s[hf][nt][e], ready ? 1.f : sc_f[nt][e & 1], ready ? 0.f : kPUp - m[nt][e & 1]));
                    l[nt][0] += w[0] + w[2];
                    l[nt][1] += w[1] + w[3];
                    pb[nt][0] = transpose_8x8(pack_f16x2(w[0], w[1]));
                    pb[nt][1] = transpose_8x8(pack_f16x2(w[2], w[3]));
                }
                with_values(hf, [&](int i, const uint32_t (&a)[4]) {
#pragma unroll
                    for (int nt = 0; nt < kNT; ++nt) mma_f16_16816(o[nt][i], a, pb[nt][0], pb[nt][1]);
                });
            }
        }

        // ---- the warps' states become one (warp 0's)
#pragma unroll
        for (int nt = 0; nt < kNT; ++nt)
#pragma unroll
            for (int e = 0; e < 2; ++e)
#pragma unroll
                for (int off = 4; off < 32; off <<= 1) l[nt][e] += __shfl_xor_sync(0xffffffffu, l[nt][e], off);
        float4* s_ml = s_fold + F::kWarps / 2 * kNT * 8 * 32;
#pragma unroll
        for (int half = F::kWarps / 2; half > 0; half >>= 1) {
            __syncthreads();
            const int at = warp % half;
            if (warp >= half && warp < 2 * half) {
#pragma unroll
                for (int nt = 0; nt < kNT; ++nt) {
#pragma unroll
                    for (int i = 0; i < 8; ++i)
                        s_fold[((at * kNT + nt) * 8 + i) * 32 + lane] =
                            make_float4(o[nt][i][0], o[nt][i][1], o[nt][i][2], o[nt][i][3]);
                    s_ml[(at * kNT + nt) * 32 + lane] = make_float4(m[nt][0], m[nt][1], l[nt][0], l[nt][1]);
                }
            }
            __syncthreads();
            if (warp < half) {
#pragma unroll
                for (int nt = 0; nt < kNT; ++nt) {
                    const float4 ml = s_ml[(at * kNT + nt) * 32 + lane];
                    const float om[2] = {ml.x, ml.y}, ol[2] = {ml.z, ml.w};
                    float a[2], b[2];
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const float top = fmaxf(m[nt][e], om[e]), base = top == kNegInf ? 0.f : top;
                        a[e] = ex2(m[nt][e] - base);
                        b[e] = ex2(om[e] - base);
                        l[nt][e] = l[nt][e] * a[e] + ol[e] * b[e];
                        m[nt][e] = top;
                    }
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const float4 v = s_fold[((at * kNT + nt) * 8 + i) * 32 + lane];
                        o[nt][i][0] = o[nt][i][0] * a[0] + v.x * b[0];
                        o[nt][i][1] = o[nt][i][1] * a[1] + v.y * b[1];
                        o[nt][i][2] = o[nt][i][2] * a[0] + v.z * b[0];
                        o[nt][i][3] = o[nt][i][3] * a[1] + v.w * b[1];
                    }
                }
            }
        }
        const bool whole = n == cur.T;
        if (warp == 0) {
            const float vh = p.v_head ? __ldcg(p.v_head + cur.h) : 1.f;
            const int slot = 2 * cta + (first_piece ? 0 : 1);
#pragma unroll
            for (int nt = 0; nt < kNT; ++nt)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const int row = nt * 8 + 2 * c + e;
                    if (row >= p.n_rows) continue;
                    const float inv = l[nt][e] > 0.f ? vh / l[nt][e] : l[nt][e] == 0.f ? 0.f : l[nt][e];   // (NaN stays)
                    if (whole) {
                        const int i = s_draft[row];
                        uint2* dst = reinterpret_cast<uint2*>(
                            p.out + (((size_t)bg * p.R + i) * p.Hq + (size_t)cur.h * p.G + (row - i * p.G)) * kPackDim + 16 * r);
#pragma unroll
                        for (int i2 = 0; i2 < 4; ++i2)
                            dst[i2] = make_uint2(pack_bf16x2(o[nt][2 * i2][e] * inv, o[nt][2 * i2][e + 2] * inv),
                                                 pack_bf16x2(o[nt][2 * i2 + 1][e] * inv, o[nt][2 * i2 + 1][e + 2] * inv));
                    } else {
                        float4* dst = reinterpret_cast<float4*>(p.part_o + ((size_t)slot * p.n_rows + row) * kPackDim + 16 * r);
#pragma unroll
                        for (int i2 = 0; i2 < 4; ++i2)
                            dst[i2] = make_float4(o[nt][2 * i2][e] * inv, o[nt][2 * i2][e + 2] * inv,
                                                  o[nt][2 * i2 + 1][e] * inv, o[nt][2 * i2 + 1][e + 2] * inv);
                        if (r == 0) p.part_ml[(size_t)slot * p.n_rows + row] = make_float2(m[nt][e], l[nt][e]);
                    }
                }
            // a cut span that starts here: its last tile's owner ends its pieces.
            // This share's last unit is that of its last tile, so the span's
            // last tile lies T - (cur.t + n) units past it.
            if (threadIdx.x == 0 && !whole && cur.t == 0) {
                const long long last = first_unit(cta + 1, U, Gc) - 1 + (cur.T - n);
                p.jobs[cta] = Job{bg, cur.h, slot, owner_of(last, U, Gc) - cta + 1};
            }
        }
        done += n;
        cur.t += n - 1;
        advance(cur, s_len, nb, p.n_spans, F::kTile);
        first_piece = false;
        __syncthreads();   // the query rows and the fold's room are free again
    }
    cp_async_wait<0>();
}

#include "packed_attention_tc.cuh"

// ---------------------------------------------------------------------------
// Joins the pieces of the span that starts in CTA c of the main kernel (if one
// does): o = sum_j w_j o_j with w_j = l_j 2^(m_j - M) / sum, a warp for a row.
// ---------------------------------------------------------------------------
constexpr int kMergeThreads = 256;
constexpr int kMergeRows = kMergeThreads / 32;
constexpr int kMergePieces = 8;   // pieces requested together

__global__ void __launch_bounds__(kMergeThreads) packed_merge_kernel(const PackedAttnParams p) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    wait_prior_grid();
    allow_dependent_launch();
    const int4 jv = __ldcg(reinterpret_cast<const int4*>(p.jobs + blockIdx.x));
    const Job job{jv.x, jv.y, jv.z, jv.w};
    if (job.n < 2) return;
    auto slot = [&](int j) { return (size_t)(j == 0 ? job.slot0 : 2 * ((int)blockIdx.x + j)); };
    for (int row = blockIdx.y * kMergeRows + warp; row < p.n_rows; row += gridDim.y * kMergeRows) {
        float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
        float M = kNegInf, sum = 0.f;
        for (int j0 = 0; j0 < job.n; j0 += kMergePieces) {
            float4 v[kMergePieces];
            float2 ml[kMergePieces];
#pragma unroll
            for (int j = 0; j < kMergePieces; ++j) {
                ml[j] = make_float2(kNegInf, 0.f);
                v[j] = make_float4(0.f, 0.f, 0.f, 0.f);
                if (j0 + j < job.n) {
                    const size_t at = slot(j0 + j) * p.n_rows + row;
                    ml[j] = __ldcg(p.part_ml + at);
                    v[j] = __ldcg(reinterpret_cast<const float4*>(p.part_o + at * kPackDim) + lane);
                }
            }
            float top = M;
#pragma unroll
            for (int j = 0; j < kMergePieces; ++j) top = fmaxf(top, ml[j].x);
            const float base = top == kNegInf ? 0.f : top, keep = ex2(M - base);
            M = top;
            sum *= keep;
            acc.x *= keep;
            acc.y *= keep;
            acc.z *= keep;
            acc.w *= keep;
#pragma unroll
            for (int j = 0; j < kMergePieces; ++j) {
                const float w = ml[j].y * ex2(ml[j].x - base);   // (0 for a piece without a key)
                sum += w;
                acc.x = fmaf(w, v[j].x, acc.x);
                acc.y = fmaf(w, v[j].y, acc.y);
                acc.z = fmaf(w, v[j].z, acc.z);
                acc.w = fmaf(w, v[j].w, acc.w);
            }
        }
        const float inv = sum > 0.f ? 1.f / sum : sum == 0.f ? 0.f : sum;
        const int head = job.h / p.n_rb, of = (job.h - head * p.n_rb) * p.n_rows + row, i = of / p.G;
        if (of >= p.n_all) continue;
        uint2* dst = reinterpret_cast<uint2*>(
            p.out + (((size_t)job.b * p.R + i) * p.Hq + (size_t)head * p.G + (of - i * p.G)) * kPackDim + 4 * lane);
        *dst = make_uint2(pack_bf16x2(acc.x * inv, acc.y * inv), pack_bf16x2(acc.z * inv, acc.w * inv));
    }
}

size_t align256(size_t n) { return (n + 255) & ~size_t(255); }

using Kernel = void (*)(const PackedAttnParams);
struct Choice {
    Kernel kern;
    int threads, smem;
    int blocks;   // of an SM, where the occupancy query is not asked; 0: it is
};
template <int kNT>
Choice choice() {
    return {packed_attention_kernel<kNT>, Form<kNT>::kThreads, Form<kNT>::kSmem, 0};
}
template <int kN>
Choice choice_tc() {
    return {packed_attention_tc_kernel<kN>, TcForm<kN>::kThreads, TcForm<kN>::kSmem, 1};
}
constexpr int kForms = 7;

// The form for a number of query rows of a span: up to 24 the one above (24 rows, 64
// requests of 4096 keys, 8 KV heads: 128 us, 138 in the tcgen05 form), from 25 on the
// tcgen05 form (28 rows: 138 us, 170 in the other one).
int form_of(int rows) {
    return rows <= 24 ? (rows + 7) / 8 - 1 : rows <= 32 ? 3 : rows <= 48 ? 4 : rows <= 64 ? 5 : 6;
}
Choice choice_of(int form) {
    static const Choice all[kForms] = {choice<1>(), choice<2>(), choice<3>(), choice_tc<32>(), choice_tc<48>(), choice_tc<64>(),
                                       choice_tc<80>()};
    return all[form];
}

// CTAs of a form that an SM holds at once (kept for each device), the limit of
// dynamic shared memory set on the way.
int resident_of(int form) {
    static std::atomic<int> kept[64][kForms];
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) {
        cudaGetLastError();
        return 0;
    }
    if (!kept[dev][form]) {
        const Choice c = choice_of(form);
        int n = 0;
        if (cudaFuncSetAttribute(c.kern, cudaFuncAttributeMaxDynamicSharedMemorySize, c.smem) != cudaSuccess ||
            cudaOccupancyMaxActiveBlocksPerMultiprocessor(&n, c.kern, c.threads, c.smem) != cudaSuccess || n <= 0) {
            cudaGetLastError();
            return 0;
        }
        // (the query answers 1 for a kernel that allocates tensor memory, whatever
        // it allocates)
        if (c.blocks) n = c.blocks;
        kept[dev][form] = n;
    }
    return kept[dev][form];
}

// Workspace: the status word (256 B), the jobs, then the pieces' (maximum, sum) and outputs.
struct PackedPlan {
    int form, n_all, n_rb, rows, grid;
    size_t off_ml, off_o, bytes;
};
PackedPlan plan_packed(const cs_attn_dims& d, int rows, int sm_count) {
    PackedPlan pl{};
    pl.n_all = rows * (d.n_q_heads / d.n_kv_heads);
    // more rows than the widest form's in blocks of equal size, each reading and decoding
    // the keys again (64 requests of 4096 keys, 8 KV heads: 80 rows 186 us, 88 288, 136 344,
    // where the bytes take 44; before the tcgen05 form's later steps 136 rows took 519 us in
    // two blocks, 870 in one of the other form)
    pl.n_rb = (pl.n_all + kTcMaxRows - 1) / kTcMaxRows;
    pl.rows = (pl.n_all + pl.n_rb - 1) / pl.n_rb;
    pl.form = form_of(pl.rows);
    const int res = resident_of(pl.form);
    pl.grid = sm_count * (res > 0 ? res : 1);
    if (pl.grid > kMaxGrid) pl.grid = kMaxGrid;
    pl.off_ml = 256 + align256(sizeof(Job) * (size_t)pl.grid);
    pl.off_o = pl.off_ml + align256(sizeof(float2) * 2 * (size_t)pl.grid * pl.rows);
    pl.bytes = pl.off_o + align256(sizeof(float) * kPackDim * 2 * (size_t)pl.grid * pl.rows);
    return pl;
}

}  // namespace

size_t packed_attention_workspace_bytes(const cs_attn_dims& d, int rows, int sm_count) {
    return plan_packed(d, rows, sm_count).bytes;
}

cs_status launch_packed_attention(const cs_attn_dims& d, const void* q, const cs_packed_pool& pool,
                                  const int32_t* page_table, const int32_t* ctx_lens, int rows, void* out,
                                  void* workspace, cudaStream_t stream) {
    const PackedPlan pl = plan_packed(d, rows, current_sm_count());
    uint8_t* ws = static_cast<uint8_t*>(workspace);
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
    p.status = reinterpret_cast<int*>(ws);
    p.jobs = reinterpret_cast<Job*>(ws + 256);
    p.part_ml = reinterpret_cast<float2*>(ws + pl.off_ml);
    p.part_o = reinterpret_cast<float*>(ws + pl.off_o);
    p.Hq = d.n_q_heads;
    p.Hkv = d.n_kv_heads;
    p.G = d.n_q_heads / d.n_kv_heads;
    p.R = rows;
    p.n_rows = pl.rows;
    p.n_all = pl.n_all;
    p.n_rb = pl.n_rb;
    p.n_spans = d.n_kv_heads * pl.n_rb;
    p.ps = d.page_size;
    while ((1 << p.ps_log2) < d.page_size) ++p.ps_log2;
    p.max_pages = d.max_pages_per_seq;
    p.P = d.num_pages;
    p.span_x = 1;
    p.scale_log2 = (d.sm_scale > 0.f ? d.sm_scale : 1.0f / sqrtf((float)d.head_dim)) * 1.4426950408889634f;
    const Choice k = choice_of(pl.form);
    if (resident_of(pl.form) <= 0) return fail(CS_ERR_CUDA, "packed_attention_kernel does not fit this device");
    const unsigned chunks = (unsigned)((pl.rows + kMergeRows - 1) / kMergeRows);
    for (int b0 = 0; b0 < d.batch; b0 += kMaxBatchPerLaunch) {
        p.b_base = b0;
        p.n_batch = d.batch - b0 < kMaxBatchPerLaunch ? d.batch - b0 : kMaxBatchPerLaunch;
        cudaError_t e = launch_dependent(k.kern, dim3(pl.grid), dim3(k.threads), (size_t)k.smem, stream, p);
        if (e != cudaSuccess) return cuda_fail(e, "packed_attention_kernel launch");
        e = launch_dependent(packed_merge_kernel, dim3(pl.grid, chunks), dim3(kMergeThreads), 0, stream, p);
        if (e != cudaSuccess) return cuda_fail(e, "packed_merge_kernel launch");
    }
    return CS_OK;
}

}  // namespace cs
