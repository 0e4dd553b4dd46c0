// chunk_attention.cu -- attention of every request's newest tokens over the paged
// bf16 cache, causal among them (cs_chunk_attention; the formula is in cachespec.h).
//
// Work.  The query rows of a request and KV head (row r: token r / G, query head
// h G + r % G) are cut into blocks of whole tokens, up to 256 rows, and a block's
// keys into tiles of 128.  A block weighs its keys and what it costs to begin and
// end one; a persistent grid of one CTA an SM takes equal contiguous ranges of the
// whole weight, whatever the requests' sizes: blocks are cut between tiles where the
// ranges end, and the CTA that comes to the end of a cut block's pieces last joins them.
// The weights have closed forms, so a CTA finds its range, and who has the rest of a
// block, from the lengths alone.
//
// A CTA (twenty warps):
//   warps 4-19      softmax, of query rows 0-127 and then 128-255 of a tile: a warp takes
//                   16 rows and half of a tile's keys, two threads a row;
//   warps 0, 3      issue the products of either: S = Q K^T (M 128, N 128 keys, 8 steps of 16
//                   dims) and O += P V (N 128 dims, 8 steps of 16 keys for either term of P),
//                   tcgen05 with S, P (over S) and O in tensor memory: 2 x (128 + 128) columns;
//   warp 1          brings K and V tiles (TMA, one box a page piece) into a ring of
//                   five 32 KB stages;
//   warp 2          brings a block's query rows (TMA).
// The products of one half run while the softmax of the other does, and a half's S of
// the next tile being complete says that P V of this one is too (a thread's products
// complete in order), so O may be rescaled then.  The running maximum moves only for a
// growth of more than 2^8.  Either query tile has an issuing warp of its own: the queue of
// products is short, and what one warp does between its products showed (with one term of
// P, 4096 tokens over 12288, 64 / 8 heads: 1270 us with one, 1189 with two).
// P is the sum of two bf16 terms, as in verify attention: one alone leaves 2e-3 + 1e-2 |out|
// in rows of few keys whose values cancel, and adds 1.5e-3 to an output's error everywhere,
// where its own rounding is 1.7e-3 (2-norms).  The second term is half as much again of
// products (the same case: 1550-1620 us, 1190 without it; prompts of 129 to 1024 tokens, 32
// heads each: 128 and 111; single tokens over contexts to 8192: 385 and 372).  Skipping it
// where every weight is small against its row's sum so far gave 1335-1400 in the first of
// these, but 137 in the second, and 117 instead of 108 in mixed batches: what decides it
// stands between the scores and the weights.
// Every wait on a barrier is bounded; one that gives up sets the status word.
//
// What bounds it: the products of a tile of 256 rows and 128 keys, 3 x 1024 cycles; in the first
// case above all of them come at 1.8 PFLOP/s, what a library product has here.  Single tokens
// over long contexts: the memory (128 requests, contexts to 8192: 6.4 TB/s), and the chain of
// a tile of one query tile.  Short calls: their start (5 us to the first tile), 4.2 us a
// block, and how even the ranges are.
#include <cudaTypedefs.h>
#include <math.h>

#include <algorithm>
#include <atomic>

#include "cs_internal.h"
#include "ragged.cuh"

namespace cs {
namespace {

constexpr int kD = 128;
constexpr int kRows = 256;                         // query rows of a block
constexpr int kHalf = 128;                         // ... of one of its two MMA tiles
constexpr int kKeys = 128;                         // keys of a tile
constexpr int kThreads = 640;
constexpr int kMmaWarp = 0, kKvWarp = 1, kQWarp = 2, kFirstSoftmax = 4;   // (warp 3: products)
constexpr int kStages = 5;
constexpr int kTileBytes = kKeys * kD * 2;
constexpr int kQBytes = kRows * kD * 2;
constexpr int kSmem = kQBytes + kStages * kTileBytes;
constexpr int kSmallQRows = 32;                    // blocks of few rows bring in no more than these
// What beginning and ending a block costs, in keys (pieces of 256 rows take 4.2 us and 2 a
// tile; 208 instead: 8 prompts 129 us, 127 so).
constexpr int kBeginKeys = 288;
// A range's end moves by so many keys, and so many a row, to a block's beginning or end; a
// call whose page table holds no more than kUncut keys a row has no cuts.  A cut costs its two
// CTAs 4 and 7 us for 252 rows.  (24 requests, four of 301-512 new tokens: 107 us; with 384
// and 2 a row either way 110; with 352, 64 and none a row 108, but 777 tokens 27 for 19.  One
// token over 1023, 4095 keys: 12.5 and 16.0 us; with 400 to the end too 18 and 21; over 512
// keys in pieces 10.9, 10.5 whole.  Where the table is wider, leaving contexts of up to kUncut
// keys whole was no gain: over 512 keys 12.2, 11.3 so; 8 requests of 400 13.4, 15.0 so.)
constexpr int kCutKeys = 400, kCutBack = 128, kCutRow = 1, kUncut = 640;
static_assert(kCutKeys + kCutRow >= kBeginKeys + kKeys / 2 && kCutBack >= kKeys / 2, "every piece of a cut block has a tile");
constexpr int kLeast = 192, kLeastRow = 2;         // a CTA's share where blocks are few: so many keys, and so many a row
constexpr int kMaxBatch = 1024;                    // requests of a launch
constexpr float kMostOver = 8.f - kPShift;         // weights are at most 2^8 times 2^-kPShift

struct ChunkParams {
    RaggedBatch batch;
    const int32_t* page_table;
    __nv_bfloat16* out;
    int* status;
    // cut blocks, by the CTA that one begins in: how many of its tiles are done (0 between
    // calls); and of their pieces, by the CTA, the one that it goes on with and the one that
    // it begins: rows' maxima (in powers of two) and sums, and outputs divided by the sums
    int* done;                 // [grid]
    // or, where a second kernel joins them: first row of q, KV head, tokens, flags
    int4* slots;               // [2 grid]
    float2* part_ml;           // [2 grid, rows]
    float* part_o;             // [2 grid, rows, 128]
    int b0, nb;                // requests of this launch
    int Hq, Hkv, G, ps, ps_log2, max_pages, P;
    int block_tokens;          // whole tokens of a block
    int small_tokens;          // ... of the small query box
    int rows;                  // rows of a slot
    bool join_here;            // the last to come joins a block's pieces
    int cut_back;              // see moved()
    int least;                 // of a CTA's share, 0: whatever it is
    HostDivisor by_block, by_grid;   // quotients by block_tokens, by the grid
    float scale_log2;
};
constexpr int kUsed = 1, kEnds = 2;                // flags of a slot: it holds a piece, which has its block's last tile
constexpr int kJoinBlocks = 2;                     // at least grid / 2 blocks: they are joined in the kernel

// Weights are W: 32 bits where the whole of a call's is sure to fit (the schedule is
// then half as long), else 64.
__device__ __forceinline__ uint32_t quotient(uint32_t a, uint32_t b) { return a / b; }
__device__ __forceinline__ uint64_t quotient(uint64_t a, uint64_t b) { return (uint64_t)div_pos((long long)a, (long long)b); }

// A request's blocks: block i has tokens [i T, min(n, (i+1) T)) and the keys in front
// of and at the last of them; it weighs its keys + kBeginKeys.
template <typename W>
struct Blocks {
    int n, L, T, count;
    __device__ __forceinline__ Blocks(int n_, int L_, const HostDivisor& T_)
        : n(n_), L(L_), T((int)T_.d), count((int)T_((uint32_t)n_ + T_.d - 1)) {}
    // the weight of blocks 0 .. i-1
    __device__ __forceinline__ W before(int i) const {
        const int first = L - n;   // keys in front of the new tokens
        const int full = min(i, count - 1);
        // blocks without a key (more new tokens than keys): all in front
        const int none = first < 0 ? min(full, -first / T) : 0;
        const W a = none, b = full;
        W w = (b - a) * (W)(long long)first + T * ((b * (b + 1) - a * (a + 1)) / 2) + b * kBeginKeys;
        if (i == count) w += L + kBeginKeys;
        return w;
    }
    // the block that place x of the whole weight lies in
    __device__ __forceinline__ int at(W x) const {
        // i (a + T / 2) + i^2 T / 2 = x, nearly; then exactly
        const float a = (float)(L - n) + kBeginKeys + 0.5f * (float)T, y = (float)x;
        int i = L < n ? 0 : (int)(2.f * y / (a + sqrtf(a * a + 2.f * (float)T * y)));
        i = max(0, min(i, count - 1));
        while (i > 0 && before(i) > x) --i;
        while (i + 1 < count && before(i + 1) <= x) ++i;
        return i;
    }
};

// The tile at place x of a block's weight w = keys + kBeginKeys
__device__ __forceinline__ int tile_at(int x, int keys) {
    const int tiles = (keys + kKeys - 1) / kKeys;
    if (x <= 0) return 0;
    if (x >= keys + kBeginKeys) return tiles;
    return min(tiles, max(0, x - kBeginKeys + kKeys / 2) / kKeys);
}

// Where a range's end at place x of a block's weight w moves: to an end of the block that
// is near.  (A cut block's pieces but one are written and read again in fp32, and rows are
// what that costs.  In front a block's beginning counts too.)
__device__ __forceinline__ int moved(int x, int w, int rows, int back) {
    const bool early = x <= kCutKeys + kCutRow * rows, late = w - x <= back + kCutRow * rows;
    return early && (!late || 2 * x <= w) ? 0 : late ? w : x;
}

// The ends of the ranges inside one block: its beginning in the whole weight, its weight
// and rows; equal ranges of `each`, the first `over` of them by one more.
template <typename W>
struct Cuts {
    W x0, each;
    int w, rows;
    int over, ctas, back;
    // where CTA c's range begins in the block (0, w: in front of it, behind it)
    __device__ __forceinline__ int begin_of(int c) const {
        const W x = each * c + min(c, over);
        return x <= x0 ? 0 : x - x0 >= (W)w ? w : moved((int)(x - x0), w, rows, back);
    }
    // the CTA that the block begins in
    __device__ __forceinline__ int first() const {
        const W more = (each + 1) * over;
        const W at = x0 < more ? quotient(x0, each + 1) : over + quotient(x0 - more, each);
        // (where starts decrease the weights may not fit: still one of the grid)
        int c = at < (W)ctas ? (int)at : ctas - 1;
        while (c + 1 < ctas && begin_of(c + 1) == 0) ++c;
        return c;
    }
};

// Where a CTA's range begins.
struct Begin {
    int b, h, i, count;        // request of the launch, KV head, block of as many
    int start, n, L;           // the request's rows and length
    int off;                   // how far into the block's weight
};

// One piece after the other of a CTA's range; every warp goes through them by itself.
template <typename W>
struct Pieces {
    const ChunkParams& p;
    Begin at;                  // where the next piece begins
    W left;                    // what is left of the range
    // the piece: tiles [t0, t1) of `tiles`, the block's keys and tokens, its request, KV
    // head and place
    int t0, t1, tiles, keys, token0, tokens;
    int b, h, L, start;
    int off, end;              // its part of the block's weight

    __device__ __forceinline__ Pieces(const ChunkParams& p_, const Begin& begin, W size)
        : p(p_), at(begin), left(begin.b >= 0 ? size : 0) {}
    // false: no more
    __device__ __forceinline__ bool next() {
        while (left > 0) {
            token0 = at.i * p.block_tokens;
            tokens = min(at.n - token0, p.block_tokens);
            keys = max(0, at.L - at.n + token0 + tokens);
            tiles = (keys + kKeys - 1) / kKeys;
            const int w = keys + kBeginKeys - at.off, take = left < (W)w ? (int)left : w;
            t0 = tile_at(at.off, keys);
            t1 = tile_at(at.off + take, keys);
            const bool there = t1 > t0 || (tiles == 0 && at.off == 0);
            b = p.b0 + at.b;
            h = at.h;
            L = at.L;
            start = at.start;
            off = at.off;
            end = at.off + take;
            left -= take;
            at.off = 0;
            if (left > 0 && ++at.i == at.count) {
                at.i = 0;
                if (++at.h == p.Hkv) {
                    at.h = 0;
                    at.n = 0;
                    while (at.n == 0 && ++at.b < p.nb) p.batch.rows_of(p.b0 + at.b, at.start, at.n, at.L);
                    at.count = (int)p.by_block((uint32_t)at.n + p.by_block.d - 1);
                    if (at.b >= p.nb) left = 0;
                }
            }
            if (there) return true;
        }
        return false;
    }
};

// ------------------------------------------------------------- tensor memory
// All of these are a whole warp's at once: after threads went ways of their own, and after
// a barrier.cta (which does not bring a warp together), __syncwarp() comes first.
// 16 lanes, twice: threads 0-15 have lanes l .. l+15 of the address at its columns,
// threads 16-31 the same lanes kSplit columns on (32 or 16 columns a thread).
template <int kSplit>
__device__ __forceinline__ void tmem_ld32(uint32_t addr, float (&v)[32]) {
    uint32_t r[32];
    asm volatile(
        "tcgen05.ld.sync.aligned.16x32bx2.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,"
        "%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32], %33;"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
          "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]),
          "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]),
          "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]),
          "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
        : "r"(addr), "n"(kSplit));
#pragma unroll
    for (int i = 0; i < 32; ++i) v[i] = __uint_as_float(r[i]);
}
template <int kSplit>
__device__ __forceinline__ void tmem_ld16(uint32_t addr, uint32_t (&r)[16]) {
    asm volatile(
        "tcgen05.ld.sync.aligned.16x32bx2.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16], %17;"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
          "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
        : "r"(addr), "n"(kSplit));
}
template <int kSplit>
__device__ __forceinline__ void tmem_st16(uint32_t addr, const uint32_t (&r)[16]) {
    asm volatile(
        "tcgen05.st.sync.aligned.16x32bx2.x16.b32 [%0], %1, {%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17};" ::"r"(
            addr),
        "n"(kSplit), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]),
        "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
        : "memory");
}
// Waits for the loads so far; the values go through it, so that nothing that uses them
// moves in front of it.
__device__ __forceinline__ void tmem_ld_done(float (&v)[32]) {
    asm volatile("tcgen05.wait::ld.sync.aligned;"
                 : "+f"(v[0]), "+f"(v[1]), "+f"(v[2]), "+f"(v[3]), "+f"(v[4]), "+f"(v[5]), "+f"(v[6]), "+f"(v[7]),
                   "+f"(v[8]), "+f"(v[9]), "+f"(v[10]), "+f"(v[11]), "+f"(v[12]), "+f"(v[13]), "+f"(v[14]),
                   "+f"(v[15]), "+f"(v[16]), "+f"(v[17]), "+f"(v[18]), "+f"(v[19]), "+f"(v[20]), "+f"(v[21]),
                   "+f"(v[22]), "+f"(v[23]), "+f"(v[24]), "+f"(v[25]), "+f"(v[26]), "+f"(v[27]), "+f"(v[28]),
                   "+f"(v[29]), "+f"(v[30]), "+f"(v[31])
                 :: "memory");
}
__device__ __forceinline__ void tmem_ld_done(uint32_t (&v)[16]) {
    asm volatile("tcgen05.wait::ld.sync.aligned;"
                 : "+r"(v[0]), "+r"(v[1]), "+r"(v[2]), "+r"(v[3]), "+r"(v[4]), "+r"(v[5]), "+r"(v[6]), "+r"(v[7]),
                   "+r"(v[8]), "+r"(v[9]), "+r"(v[10]), "+r"(v[11]), "+r"(v[12]), "+r"(v[13]), "+r"(v[14]), "+r"(v[15])
                 :: "memory");
}
__device__ __forceinline__ void tmem_st_done() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }

// D[128 x n] (+)= A B, both in shared memory
__device__ __forceinline__ void mma_ss(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t acc) {
    asm volatile(
        "{\n\t.reg .pred q;\n\tsetp.ne.b32 q, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, q;\n\t}\n" ::"r"(d),
        "l"(a), "l"(b), "r"(idesc), "r"(acc)
        : "memory");
}

// Shared-memory operands with a 128-byte swizzle, in groups of 8 rows of 128 bytes:
// query rows [dim half][row][64 dims], K-major, groups 1024 bytes apart;
__device__ __forceinline__ uint64_t q_desc(uint32_t addr) {
    return (uint64_t)((addr >> 4) & 0x3FFF) | ((uint64_t)1 << 16) | ((uint64_t)(1024 >> 4) << 32) | (1ull << 46) | (2ull << 61);
}
// K and V tiles [8-key group][dim half][key][64 dims], groups 2048 bytes apart: K
// K-major, V MN-major (its dim halves 1024 bytes apart).
__device__ __forceinline__ uint64_t k_desc(uint32_t addr) {
    return (uint64_t)((addr >> 4) & 0x3FFF) | ((uint64_t)1 << 16) | ((uint64_t)(2048 >> 4) << 32) | (1ull << 46) | (2ull << 61);
}
__device__ __forceinline__ uint64_t v_desc(uint32_t addr) {
    return (uint64_t)((addr >> 4) & 0x3FFF) | ((uint64_t)(1024 >> 4) << 16) | ((uint64_t)(2048 >> 4) << 32) | (1ull << 46) |
           (2ull << 61);
}
// bf16 operands, fp32 sums, M = N = 128; b_mn: B's N index is the contiguous one
__host__ __device__ constexpr uint32_t idesc_of(bool b_mn) {
    return (1u << 4) | (1u << 7) | (1u << 10) | (b_mn ? (1u << 16) : 0u) | ((128u >> 3) << 17) | ((128u >> 4) << 24);
}

__device__ __forceinline__ void tma_load_3d(uint32_t dst, const CUtensorMap* map, uint64_t* bar, int c0, int c1, int c2) {
    asm volatile(
        "cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes"
        " [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(dst),
        "l"(reinterpret_cast<uint64_t>(map)), "r"(c0), "r"(c1), "r"(c2), "r"(smem_u32(bar))
        : "memory");
}
__device__ __forceinline__ float max3(float a, float b, float c) {
    float d;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
    return d;
}
// Keys from lim on are hidden.
__device__ __forceinline__ void hide(float (&s)[32], int lim) {
    if (lim < 32) {
#pragma unroll
        for (int e = 0; e < 32; ++e)
            if (e >= lim) s[e] = kNegInf;
    }
}
__device__ __forceinline__ float top_of(const float (&s)[32]) {
    float a[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) a[j] = max3(s[j], s[j + 4], s[j + 8]);
#pragma unroll
    for (int e = 12; e < 28; e += 8)
#pragma unroll
        for (int j = 0; j < 4; ++j) a[j] = max3(a[j], s[e + j], s[e + 4 + j]);
#pragma unroll
    for (int j = 0; j < 4; ++j) a[j] = fmaxf(a[j], s[28 + j]);
    return fmaxf(max3(a[0], a[1], a[2]), a[3]);
}
// 1 / x, within an ulp
__device__ __forceinline__ float rcp(float x) {
    float y;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// Of a count that CTAs hand on what they wrote by
__device__ __forceinline__ int load_acquire(const int* p) {
    int x;
    asm volatile("ld.acquire.gpu.global.s32 %0, [%1];" : "=r"(x) : "l"(p) : "memory");
    return x;
}
__device__ __forceinline__ int add_acq_rel(int* p, int n) {
    int x;
    asm volatile("atom.add.acq_rel.gpu.global.s32 %0, [%1], %2;" : "=r"(x) : "l"(p), "r"(n) : "memory");
    return x;
}
// 32 bytes at once
__device__ __forceinline__ void store32(float* p, const uint32_t (&r)[8]) {
    asm volatile("st.global.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"l"(p), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]),
                 "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7])
                 : "memory");
}
// 32 bytes of an output, which is aligned to 16; kWide: to 32.  (8 prompts, 32 heads each: 111.0
// us at once, 114.5 as two stores, each half a sector; by a branch in the kernel 112.6.)
template <bool kWide>
__device__ __forceinline__ void store_out(__nv_bfloat16* p, const uint32_t (&r)[8]) {
    if constexpr (kWide) {
        store32(reinterpret_cast<float*>(p), r);
    } else {
        reinterpret_cast<uint4*>(p)[0] = make_uint4(r[0], r[1], r[2], r[3]);
        reinterpret_cast<uint4*>(p)[1] = make_uint4(r[4], r[5], r[6], r[7]);
    }
}

// (one lane)
__device__ __forceinline__ void wait_lane(uint64_t* bar, uint32_t parity, volatile int* dead, int* status) {
    if (!mbar_try_wait(bar, parity) && !*dead && !mbar_wait_bounded(bar, parity)) {
        *dead = 1;
        atomicOr(status, CS_DEVICE_WAIT_TIMEOUT);
    }
}

// The two warps of a pair: whether any of their threads says so; and a barrier.
__device__ __forceinline__ bool pair_any(int id, bool x) {
    uint32_t r;
    asm volatile(
        "{\n\t.reg .pred p, q;\n\tsetp.ne.u32 p, %1, 0;\n\t"
        "barrier.cta.red.or.pred q, %2, 64, p;\n\tselp.u32 %0, 1, 0, q;\n\t}"
        : "=r"(r)
        : "r"((uint32_t)x), "r"(id)
        : "memory");
    return r != 0;
}
// All softmax warps.
__device__ __forceinline__ void all_sync() { asm volatile("barrier.cta.sync 9, 512;" ::: "memory"); }
__device__ __forceinline__ void pair_sync(int id) { asm volatile("barrier.cta.sync %0, 64;" ::"r"(id) : "memory"); }

struct Bars {
    uint64_t kv_full[kStages], kv_empty[kStages];
    uint64_t q_full, q_empty;
    uint64_t s_full[2], p_full[2], o_full[2], o_empty[2];
    uint64_t drained;
};

// Whether no wait of the block has given up, the same answer in the whole warp.
__device__ __forceinline__ bool alive(volatile int* dead) { return !__any_sync(0xffffffffu, *dead); }

// Waits for the phase of the given parity, the whole warp; any wait returns at once
// after one of the block has given up.  (What follows then works on whatever is there,
// within the same bounds, to the end, and the status says so: no warp leaves before
// another that it meets at a barrier.)
__device__ __forceinline__ void wait(uint64_t* bar, uint32_t parity, volatile int* dead, int* status) {
    if (!mbar_try_wait(bar, parity) && !*dead && !mbar_wait_bounded(bar, parity)) {
        *dead = 1;
        atomicOr(status, CS_DEVICE_WAIT_TIMEOUT);
    }
    __syncwarp();
}

// kWide: out is aligned to 32 bytes
template <typename W, bool kWide>
__global__ void __launch_bounds__(kThreads, 1)
chunk_attention_kernel(const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v,
                       const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_q_small,
                       const ChunkParams p) {
    extern __shared__ __align__(1024) uint8_t smem[];
    uint8_t* const sq = smem;                      // [dim half][row][128 B]
    uint8_t* const ring = smem + kQBytes;
    __shared__ Bars bars;
    __shared__ W s_part[kThreads / 32];
    __shared__ Begin s_begin;
    __shared__ int s_move[2], s_over;
    __shared__ int s_join[2];                      // of the range's first piece, and of its last
    __shared__ W s_each, s_lo;
    // for the warp of the other keys: a warp's rows' sums of the first half; of the second,
    // and maxima before
    __shared__ float s_row[2][16][16];
    __shared__ uint32_t s_tmem;
    __shared__ volatile int s_dead;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

    if (warp == kMmaWarp) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_u32(&s_tmem)) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    if (warp == kKvWarp && lane == 0) {
        tma_prefetch_desc(&map_k);
        tma_prefetch_desc(&map_v);
    }
    if (warp == kQWarp && lane == 0) {
        tma_prefetch_desc(&map_q);
        tma_prefetch_desc(&map_q_small);
    }
    if (threadIdx.x == 3 * 32) {
        s_dead = 0;
        s_begin.b = -1;
        s_move[0] = s_move[1] = 0;
        for (int i = 0; i < kStages; ++i) {
            mbar_init(&bars.kv_full[i], 1);
            mbar_init(&bars.kv_empty[i], 2);
        }
        mbar_init(&bars.q_full, 1);
        mbar_init(&bars.q_empty, 2);
        for (int m = 0; m < 2; ++m) {
            mbar_init(&bars.s_full[m], 1);
            mbar_init(&bars.p_full[m], 16);
            mbar_init(&bars.o_full[m], 1);
            mbar_init(&bars.o_empty[m], 16);
        }
        mbar_init(&bars.drained, 2);
        fence_barrier_init();
    }
    // (rows that no block fills: zeros are cheaper to multiply than noise)
    for (int i = threadIdx.x; i < kQBytes / 16; i += kThreads) reinterpret_cast<uint4*>(sq)[i] = make_uint4(0, 0, 0, 0);
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    wait_prior_grid();
    allow_dependent_launch();

    // ---- the range: requests' weights, and their running sum.  Half of the threads look
    // for where it begins, the others for where it ends.
    constexpr int kHalfThreads = kThreads / 2, kEach = (kMaxBatch + kHalfThreads - 1) / kHalfThreads;
    const bool looks_for_end = threadIdx.x >= kHalfThreads;
    const int each_ = p.nb <= kHalfThreads ? 1 : kEach, b0 = (threadIdx.x - (looks_for_end ? kHalfThreads : 0)) * each_;
    W mine = 0;
    Begin own{-1, 0, 0, 0, 0, 0, 0, 0};
    W weight = 0;              // (of one KV head, of the last request looked at)
    auto look = [&](int b) {
        own.b = b;
        weight = 0;
        if (b >= p.nb) return;
        p.batch.rows_of(p.b0 + b, own.start, own.n, own.L);
        const Blocks<W> blocks(own.n, own.L, p.by_block);
        own.count = blocks.count;
        if (own.n > 0) weight = blocks.before(blocks.count);
    };
#pragma unroll 1
    for (int e = 0; e < each_; ++e) {
        look(b0 + e);
        mine += weight * p.Hkv;
    }
    W upto = mine;
#pragma unroll
    for (int d = 1; d < 32; d *= 2) {
        const W x = __shfl_up_sync(0xffffffffu, upto, d);
        if (lane >= d) upto += x;
    }
    if (lane == 31) s_part[warp] = upto;
    if (threadIdx.x < 2 && !p.join_here) p.slots[2 * blockIdx.x + threadIdx.x] = make_int4(0, 0, 0, 0);
    fence_before();
    __syncthreads();
    fence_after();
    const uint32_t tmem = s_tmem;
    // the warps' sums, by half
    constexpr int kWarps = kThreads / 64;
    W sums = lane < kWarps ? s_part[(looks_for_end ? kWarps : 0) + lane] : 0;
#pragma unroll
    for (int d = 1; d < 16; d *= 2) {
        const W x = __shfl_up_sync(0xffffffffu, sums, d);
        if (lane >= d) sums += x;
    }
    const W total = __shfl_sync(0xffffffffu, sums, kWarps - 1);
    const int before = warp - (looks_for_end ? kWarps : 0);
    const W front = __shfl_sync(0xffffffffu, sums, before > 0 ? before - 1 : 0);
    W at = upto - mine + (before > 0 ? front : 0);
    // the first CTAs take one more of what is over; with few blocks only as many work as
    // have a share that is worth a piece's join
    const W ctas = p.least ? min((W)gridDim.x, max((W)1, quotient(total, (W)p.least))) : gridDim.x;
    const W each = sizeof(W) == 4 && !p.least ? p.by_grid((uint32_t)total) : quotient(total, ctas);
    const int over = (int)(total - each * ctas), cta = min((int)blockIdx.x, (int)ctas);
    const W lo = each * cta + min(cta, over), hi = blockIdx.x < ctas ? lo + each + (cta < over) : lo;
    if (threadIdx.x == 0) {
        s_each = each;
        s_over = over;
        s_lo = lo;
    }
    // An end that is near one of its block's moves there (moved()), for both CTAs that it
    // parts.
    const W want = looks_for_end ? hi : lo;
    if (want >= at && want - at < mine) {
#pragma unroll 1
        for (int e = 0; e < each_; ++e) {
            if (each_ > 1) look(b0 + e);
            const W in = want - at;
            if (want >= at && in < weight * p.Hkv) {
                own.h = (int)quotient(in, weight);
                const W x = in - own.h * weight;
                const Blocks<W> blocks(own.n, own.L, p.by_block);
                own.i = blocks.at(x);
                const W front_ = blocks.before(own.i);
                own.off = (int)(x - front_);
                const int keys = max(0, own.L - own.n + min(own.n, (own.i + 1) * p.block_tokens));
                const int to = moved(own.off, keys + kBeginKeys, p.G * min(own.n - own.i * p.block_tokens, p.block_tokens), p.cut_back);
                s_move[looks_for_end] = to - own.off;
                own.off = to;
                if (!looks_for_end) s_begin = own;
                break;
            }
            at += weight * p.Hkv;
        }
    }
    __syncthreads();
    Pieces<W> pc(p, s_begin, hi + s_move[1] - (lo + s_move[0]));
    const uint32_t ring_at = smem_u32(ring);

    if (warp < kFirstSoftmax) {
        if (warp == kKvWarp) {
            // --------------------------------------------------- K and V tiles
            const int box = min(p.ps, kKeys), pieces = kKeys / box;
            uint32_t at_stage = 0;   // stages used so far
            while (pc.next()) {
                const int32_t* row = p.page_table + (size_t)pc.b * p.max_pages;
                auto page_of = [&](int t) {
                    const int key = t * kKeys + lane * box;
                    return lane < pieces && key < pc.L ? __ldcg(row + (key >> p.ps_log2)) : -1;
                };
                int page = pc.t0 < pc.t1 ? page_of(pc.t0) : -1;
                for (int t = pc.t0; t < pc.t1; ++t) {
                    const int key = t * kKeys + lane * box;
                    const int live = min(pieces, (pc.L - t * kKeys + box - 1) / box);
                    // (a page outside the pool reads as zeros, from in front of it)
                    const int group = (unsigned)page < (unsigned)p.P
                                          ? (int)(((long long)page * p.Hkv + pc.h) * (p.ps >> 3) + ((key & (p.ps - 1)) >> 3))
                                          : -(box >> 3);
                    if (t + 1 < pc.t1) page = page_of(t + 1);
#pragma unroll
                    for (int v = 0; v < 2; ++v) {
                        const uint32_t st = at_stage % kStages, round = at_stage / kStages;
                        if (round > 0) wait(&bars.kv_empty[st], (round - 1) & 1, &s_dead, p.status);
                        if (!alive(&s_dead)) break;   // (nothing more into a stage that may be in use)
                        ++at_stage;
                        if (lane == 0) mbar_arrive_expect_tx(&bars.kv_full[st], (uint32_t)live * box * (kD * 2));
                        __syncwarp();
                        if (lane < live)
                            tma_load_4d(ring_at + st * kTileBytes + lane * box * (kD * 2), v ? &map_v : &map_k,
                                        &bars.kv_full[st], 0, 0, 0, group);
                    }
                }
            }
            // no copy in flight at the end: every stage that was filled has landed
            for (uint32_t j = at_stage > kStages ? at_stage - kStages : 0; j < at_stage; ++j)
                if (!mbar_wait_bounded(&bars.kv_full[j % kStages], (j / kStages) & 1) && lane == 0)
                    atomicOr(p.status, CS_DEVICE_WAIT_TIMEOUT);
        } else if (warp == kQWarp) {
            // ------------------------------------------------------ query rows
            uint32_t piece = 0;
            while (pc.next()) {
                if (pc.tiles == 0) continue;
                if (piece > 0) wait(&bars.q_empty, (piece - 1) & 1, &s_dead, p.status);
                if (!alive(&s_dead)) break;
                ++piece;
                const bool few = pc.tokens <= p.small_tokens;
                const int box = few ? p.small_tokens : p.block_tokens;
                if (lane == 0) mbar_arrive_expect_tx(&bars.q_full, (uint32_t)box * p.G * (kD * 2));
                __syncwarp();
                if (lane < 2)
                    tma_load_3d(smem_u32(sq) + lane * (kQBytes / 2), few ? &map_q_small : &map_q, &bars.q_full, lane * 64,
                                pc.h * p.G, pc.start + pc.token0);
            }
            if (piece > 0 && !mbar_wait_bounded(&bars.q_full, (piece - 1) & 1) && lane == 0)
                atomicOr(p.status, CS_DEVICE_WAIT_TIMEOUT);
        } else {
            // -------------------------------------------------------- products
            const int m = warp == kMmaWarp ? 0 : 1;
            const uint64_t dq = q_desc(smem_u32(sq)) + (uint64_t)(m * (kHalf * 128) >> 4);
            const uint64_t dk = k_desc(ring_at), dv = v_desc(ring_at);
            const uint32_t t_s = tmem + m * 128, t_o = t_s + 256;
            constexpr uint32_t id_s = idesc_of(false), id_o = idesc_of(true);
            auto scores = [&](uint32_t st) {
                const uint64_t b = dk + (uint64_t)(st * kTileBytes >> 4);
#pragma unroll
                for (int s = 0; s < 8; ++s)
                    mma_ss(t_s, dq + (s >> 2) * (uint64_t)(kQBytes / 2 >> 4) + (s & 3) * 2,
                           b + (s >> 2) * (uint64_t)(1024 >> 4) + (s & 3) * 2, id_s, s > 0);
                tc_commit(&bars.s_full[m]);
            };
            uint32_t stage = 0, piece = 0, n_p = 0, n_o = 0;   // (as many phases as there were)
            auto need = [&](uint32_t n) { wait(&bars.kv_full[n % kStages], (n / kStages) & 1, &s_dead, p.status); };
            while (pc.next()) {
                if (pc.tiles == 0) continue;
                wait(&bars.q_full, piece & 1, &s_dead, p.status);
                ++piece;
                if (m == 1 && pc.tokens * p.G <= kHalf) {   // no row of this half
                    if (lane == 0) {
                        mbar_arrive(&bars.q_empty);
                        for (int t = 2 * (pc.t1 - pc.t0); t > 0; --t) {
                            const uint32_t n = stage++;
                            wait_lane(&bars.kv_full[n % kStages], (n / kStages) & 1, &s_dead, p.status);
                            mbar_arrive(&bars.kv_empty[n % kStages]);
                        }
                    }
                    stage = __shfl_sync(0xffffffffu, stage, 0);
                    continue;
                }
                need(stage);
                if (elect_one()) {
                    scores(stage % kStages);
                    tc_commit(&bars.kv_empty[stage % kStages]);
                    if (pc.t0 + 1 == pc.t1) tc_commit(&bars.q_empty);
                }
                __syncwarp();
                ++stage;
                if (n_o++ > 0) wait(&bars.o_empty[m], n_o & 1, &s_dead, p.status);
                for (int t = pc.t0; t < pc.t1; ++t) {
                    const bool last = t + 1 == pc.t1;
                    const uint32_t sv = stage % kStages, sk = (stage + 1) % kStages;
                    need(stage);
                    // slots past the context's end may hold any bits, and their weights are 0
                    // (either warp writes the same zeros before its products)
                    const int live = pc.L - t * kKeys;
                    if (live < kKeys) {
                        uint4* v = reinterpret_cast<uint4*>(ring + sv * kTileBytes);
                        for (int i = lane; i < kTileBytes / 16; i += 32) {
                            const int r = i >> 3;   // [group][half][key]
                            if ((r >> 4) * 8 + (r & 7) >= live) v[i] = make_uint4(0, 0, 0, 0);
                        }
                        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                        __syncwarp();
                    }
                    if (!last) need(stage + 1);
                    wait(&bars.p_full[m], n_p++ & 1, &s_dead, p.status);
                    fence_after();
                    if (elect_one()) {
                        const uint64_t b = dv + (uint64_t)(sv * kTileBytes >> 4);
#pragma unroll
                        for (int s = 0; s < 16; ++s)   // (16 keys' first terms, their second)
                            tc_mma_ts(t_o, t_s + s * 8, b + (s >> 1) * (uint64_t)(4096 >> 4), id_o, t > pc.t0 || s > 0);
                        if (last) tc_commit(&bars.o_full[m]);
                        else scores(sk);
                        tc_commit(&bars.kv_empty[sv]);
                        if (!last) tc_commit(&bars.kv_empty[sk]);
                        if (t + 2 == pc.t1) tc_commit(&bars.q_empty);
                    }
                    __syncwarp();
                    stage += last ? 1 : 2;
                }
            }
            // every product is complete before tensor memory is given back
            if (elect_one()) tc_commit(&bars.drained);
            __syncwarp();
            if (!mbar_wait_bounded(&bars.drained, 0) && lane == 0) atomicOr(p.status, CS_DEVICE_WAIT_TIMEOUT);
        }
    } else {
        // ------------------------------------------- softmax, four threads a row
        // Of these, warps w and w + 8 take lanes 32 (w % 4) + 16 (w / 4 % 2) .. of either half, the
        // first keys 0-63 of a tile, the second 64-127; threads i and i + 16 share a row,
        // 32 keys each (and as many dims of O).  A thread's weights lie over its own scores: of 16
        // keys the first terms, then the second.  The two warps agree at a barrier of their own
        // whether the maxima stand.
        const int sw = warp - kFirstSoftmax;
        const int part = (sw >> 3) * 2 + (lane >> 4);     // the thread's quarter of keys and dims
        const int lane0 = (sw & 3) * 32 + ((sw >> 2) & 1) * 16;
        const int pair = 1 + (sw & 7);
        const uint32_t t_row = tmem + ((uint32_t)lane0 << 16);
        const float c = p.scale_log2;
        int token[2], head[2];
#pragma unroll
        for (int m = 0; m < 2; ++m) {
            token[m] = (m * kHalf + lane0 + (lane & 15)) / p.G;
            head[m] = m * kHalf + lane0 + (lane & 15) - token[m] * p.G;
        }
        uint32_t n_s[2] = {0, 0}, n_o[2] = {0, 0};
        while (pc.next()) {
            const size_t out_at = ((size_t)(pc.start + pc.token0) * p.Hq + (size_t)pc.h * p.G) * kD + part * 32;
            const int halves = pc.tokens * p.G > kHalf ? 2 : 1;
            if (pc.tiles == 0) {   // no key at all
                const uint32_t zero[8] = {0, 0, 0, 0, 0, 0, 0, 0};
#pragma unroll
                for (int m = 0; m < 2; ++m)
                    if (token[m] < pc.tokens)
                        for (int j = 0; j < 2; ++j)
                            store_out<kWide>(p.out + out_at + ((size_t)token[m] * p.Hq + head[m]) * kD + j * 16, zero);
                continue;
            }
            // the maximum that the weights go by, what takes a score to its weight's exponent,
            // the sum of this thread's weights
            float m_run[2] = {kNegInf, kNegInf}, neg[2] = {0.f, 0.f}, l_run[2] = {0.f, 0.f};
            bool any[2];   // (the same in both warps of a pair)
#pragma unroll
            for (int m = 0; m < 2; ++m) any[m] = __any_sync(0xffffffffu, token[m] < pc.tokens);
            for (int t = pc.t0; t < pc.t1; ++t) {
#pragma unroll
                for (int m = 0; m < 2; ++m) {
                    if (m == halves) break;
                    wait(&bars.s_full[m], n_s[m] & 1, &s_dead, p.status);
                    ++n_s[m];
                    fence_after();
                    if (any[m]) {
                        const uint32_t t_s = t_row + m * 128, t_o = t_row + 256 + m * 128 + (sw >> 3) * 64;
                        float s[32];
                        tmem_ld32<32>(t_s + (sw >> 3) * 64, s);
                        tmem_ld_done(s);
                        // keys that the row sees, from this thread's first one on
                        const int lim = pc.keys - (pc.tokens - 1 - min(token[m], pc.tokens - 1)) - t * kKeys - part * 32;
                        if (__builtin_expect(lim < 32, 0)) hide(s, lim);
                        // The weights go by the maximum so far, unless a score of the pair's rows passes
                        // it by more than 8 (in powers of two), or there is none yet.
                        const float mh = top_of(s);
                        const bool need = !(fmaf(mh, c, neg[m]) <= kMostOver) || m_run[m] == kNegInf;
                        if (t == pc.t0 || pair_any(pair, need)) {
                            const float own = need ? mh : kNegInf;   // (the others' maxima stay)
                            const float mw = fmaxf(own, __shfl_xor_sync(0xffffffffu, own, 16));
                            pair_sync(pair);   // (what was there has been read)
                            if (lane < 16) s_row[1][sw][lane] = mw;
                            pair_sync(pair);
                            const float mt = fmaxf(m_run[m], fmaxf(mw, s_row[1][sw ^ 8][lane & 15]));
                            pair_sync(pair);
                            const float alpha = mt > m_run[m] ? ex2((m_run[m] - mt) * c) : 1.f;   // (0 where there was none)
                            m_run[m] = mt;
                            neg[m] = mt == kNegInf ? 0.f : -mt * c - kPShift;
                            l_run[m] *= alpha;
                            if (t != pc.t0) {
                                // P V of the tile before is complete (see above)
                                __syncwarp();
#pragma unroll 1
                                for (int q = 0; q < 2; ++q) {
                                    uint32_t o[16];
                                    tmem_ld16<32>(t_o + q * 16, o);
                                    tmem_ld_done(o);
#pragma unroll
                                    for (int i = 0; i < 16; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * alpha);
                                    tmem_st16<32>(t_o + q * 16, o);
                                }
                            }
                        }
                        const uint64_t c2 = f2_pack(c, c), n2 = f2_pack(neg[m], neg[m]);
                        uint64_t sums[2] = {0ull, 0ull};
                        __syncwarp();
#pragma unroll
                        for (int q = 0; q < 2; ++q) {   // 16 keys
                            uint32_t w[16];
#pragma unroll
                            for (int e = 0; e < 8; ++e) {
                                float x0, x1;
                                f2_unpack(f2_fma(f2_pack(s[16 * q + 2 * e], s[16 * q + 2 * e + 1]), c2, n2), x0, x1);
                                const float p0 = ex2(x0), p1 = ex2(x1);
                                sums[e & 1] = f2_add(sums[e & 1], f2_pack(p0, p1));
                                split_bf16x2(p0, p1, w[e], w[8 + e]);
                            }
                            tmem_st16<32>(t_s + (sw >> 3) * 64 + q * 16, w);
                        }
                        float a0, a1;
                        f2_unpack(f2_add(sums[0], sums[1]), a0, a1);
                        l_run[m] += a0 + a1;
                        if (t + 1 == pc.t1) {
                            // the row's sum in this warp, for the other, which reads it when the
                            // last products are complete
                            const float l = l_run[m] + __shfl_xor_sync(0xffffffffu, l_run[m], 16);
                            if (lane < 16) s_row[m][sw][lane] = l;
                            l_run[m] = l;
                            __syncwarp();
                        }
                        tmem_st_done();
                    }
                    fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&bars.p_full[m]);
                }
            }
            // ---- the piece's end
            if (pc.t0 == 0 && pc.t1 == pc.tiles) {
#pragma unroll
                for (int m = 0; m < 2; ++m) {
                    if (m == halves) break;
                    wait(&bars.o_full[m], n_o[m]++ & 1, &s_dead, p.status);
                    fence_after();
                    if (any[m]) {
                        const float l = l_run[m] + s_row[m][sw ^ 8][lane & 15];
                        const float inv = l > 0.f ? rcp(l) : 0.f;
                        float o[32];
                        tmem_ld32<32>(t_row + 256 + m * 128 + (sw >> 3) * 64, o);
                        tmem_ld_done(o);
                        if (token[m] < pc.tokens) {
                            __nv_bfloat16* dst = p.out + out_at + ((size_t)token[m] * p.Hq + head[m]) * kD;
#pragma unroll
                            for (int j = 0; j < 2; ++j) {
                                uint32_t r[8];
#pragma unroll
                                for (int e = 0; e < 8; ++e)
                                    r[e] = pack_bf16x2(o[16 * j + 2 * e] * inv, o[16 * j + 2 * e + 1] * inv);
                                store_out<kWide>(dst + j * 16, r);
                            }
                        }
                    }
                    fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&bars.o_empty[m]);
                }
                continue;
            }
            // A cut block's piece is left in fp32, but for the one that comes last: it joins
            // them, its own still in tensor memory, in the order of their tiles (so the result
            // does not go by who came last).
            const bool begins = pc.off == 0;   // (then it is the last piece of the CTA's range, else the first)
            const int mine = 2 * blockIdx.x + begins;
            const W x0 = begins ? s_lo + s_each + ((int)blockIdx.x < s_over) + s_move[1] - pc.end : s_lo + s_move[0] - pc.off;
            const Cuts<W> cuts{x0, s_each, pc.keys + kBeginKeys, pc.tokens * p.G, s_over, (int)gridDim.x, p.cut_back};
            const int first_cta = begins ? (int)blockIdx.x : cuts.first();
            bool join = false;
            if (p.join_here) {
                if (threadIdx.x == kFirstSoftmax * 32) {
                    s_join[begins] = load_acquire(p.done + first_cta) + pc.t1 - pc.t0 == pc.tiles;
                }
                all_sync();
                join = s_join[begins];
            } else if (threadIdx.x == kFirstSoftmax * 32) {
                p.slots[mine] = make_int4(pc.start + pc.token0, pc.h, pc.tokens, kUsed | (pc.t1 == pc.tiles ? kEnds : 0));
            }
#pragma unroll 1
            for (int again = 0;; ++again) {
#pragma unroll 1
                for (int m = 0; m < halves; ++m) {
                    if (again == 0) wait(&bars.o_full[m], (m ? n_o[1] : n_o[0]) & 1, &s_dead, p.status);
                    fence_after();
                    if (!(m ? any[1] : any[0])) continue;
                    const float l = (m ? l_run[1] : l_run[0]) + s_row[m][sw ^ 8][lane & 15];
                    const float top = m ? m_run[1] : m_run[0];
                    const float inv = l > 0.f ? rcp(l) : 0.f;
                    const int row = m * kHalf + lane0 + (lane & 15), token_ = m ? token[1] : token[0];
                    // pieces that this kernel joins: as the threads hold them, 16 rows and 64
                    // dims a warp, [4 dims][thread]
                    const size_t held = (size_t)(row >> 4) * (16 * kD) + (sw >> 3) * (8 * kD) + lane * 4;
                    const float2 ml = make_float2(top == kNegInf ? kNegInf : top * c, l);
#pragma unroll 1
                    for (int q = 0; q < 2; ++q) {   // 16 dims
                        uint32_t w[16];
                        __syncwarp();
                        tmem_ld16<32>(t_row + 256 + m * 128 + (sw >> 3) * 64 + q * 16, w);
                        tmem_ld_done(w);
                        if (token_ < pc.tokens) {
                            float o[16];
#pragma unroll
                            for (int e = 0; e < 16; ++e) o[e] = __uint_as_float(w[e]) * inv;
                            if (join) {
                                float sum[16];
                                float2 all = make_float2(kNegInf, 0.f);
#pragma unroll
                                for (int e = 0; e < 16; ++e) sum[e] = 0.f;
                                int x = 0;
#pragma unroll 1
                                for (int cta = first_cta; x < cuts.w && cta < cuts.ctas; ++cta) {
                                    const int y = cuts.begin_of(cta + 1);
                                    const bool there = tile_at(x, pc.keys) < tile_at(y, pc.keys);
                                    x = y;
                                    if (!there) continue;
                                    const int slot = 2 * cta + (cta == first_cta);
                                    const size_t at_row = (size_t)slot * p.rows + row;
                                    const float* from = p.part_o + (size_t)slot * p.rows * kD + held + q * 512;
                                    const float2 z = slot == mine ? ml : __ldcg(p.part_ml + at_row);
                                    float4 v[4];
#pragma unroll
                                    for (int j = 0; j < 4; ++j) {
                                        v[j] = make_float4(o[4 * j], o[4 * j + 1], o[4 * j + 2], o[4 * j + 3]);
                                        if (slot != mine) v[j] = __ldcg(reinterpret_cast<const float4*>(from + j * 128));
                                    }
                                    const float most = fmaxf(all.x, z.x);
                                    const float f = most == kNegInf ? 0.f : ex2(all.x - most);
                                    const float g = most == kNegInf ? 0.f : ex2(z.x - most) * z.y;
                                    all = make_float2(most, all.y * f + g);
#pragma unroll
                                    for (int j = 0; j < 4; ++j) {
                                        sum[4 * j] = fmaf(v[j].x, g, sum[4 * j] * f);
                                        sum[4 * j + 1] = fmaf(v[j].y, g, sum[4 * j + 1] * f);
                                        sum[4 * j + 2] = fmaf(v[j].z, g, sum[4 * j + 2] * f);
                                        sum[4 * j + 3] = fmaf(v[j].w, g, sum[4 * j + 3] * f);
                                    }
                                }
                                const float r = all.y > 0.f ? rcp(all.y) : 0.f;
#pragma unroll
                                for (int e = 0; e < 16; ++e) o[e] = sum[e] * r;
                                uint32_t r8[8];
#pragma unroll
                                for (int e = 0; e < 8; ++e) r8[e] = pack_bf16x2(o[2 * e], o[2 * e + 1]);
                                store_out<kWide>(p.out + out_at + ((size_t)token_ * (p.Hq - p.G) + row) * kD + q * 16, r8);
                            } else {
                                const size_t at_row = (size_t)mine * p.rows + row;
                                if (p.join_here) {
                                    float* to = p.part_o + (size_t)mine * p.rows * kD + held + q * 512;
#pragma unroll
                                    for (int j = 0; j < 4; ++j)
                                        __stcg(reinterpret_cast<float4*>(to + j * 128),
                                               make_float4(o[4 * j], o[4 * j + 1], o[4 * j + 2], o[4 * j + 3]));
                                } else {
#pragma unroll
                                    for (int j = 0; j < 2; ++j) {
                                        uint32_t r8[8];
#pragma unroll
                                        for (int e = 0; e < 8; ++e) r8[e] = __float_as_uint(o[8 * j + e]);
                                        store32(p.part_o + at_row * kD + part * 32 + q * 16 + j * 8, r8);
                                    }
                                }
                                if (part == 0 && q == 0) p.part_ml[at_row] = ml;
                            }
                        }
                    }
                }
                if (join || again || !p.join_here) break;
                all_sync();   // (with which the piece is the thread's to hand on)
                if (threadIdx.x == kFirstSoftmax * 32)
                    s_join[begins] = add_acq_rel(p.done + first_cta, pc.t1 - pc.t0) + pc.t1 - pc.t0 == pc.tiles;
                all_sync();
                join = s_join[begins];
                if (!join) break;
            }
            if (join && threadIdx.x == kFirstSoftmax * 32) p.done[first_cta] = 0;
            fence_before();
            __syncwarp();
            ++n_o[0];
            if (halves == 2) ++n_o[1];
            if (lane < halves) mbar_arrive(&bars.o_empty[lane]);
        }
    }
    fence_before();
    __syncthreads();
    fence_after();
    if (warp == kMmaWarp) {
        __syncwarp();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem) : "memory");
    }
}

// ------------------------------------------------------------------ the join
// Where blocks are few and have many pieces, CTA (c, y) joins those of the block that
// begins in main CTA c and ends in a later one, rows 16 y and on, a row a warp at a time:
// a lane a piece for the weights, then the outputs weighted by them, four on their way
// at once.  (Four warps of 32 registers and no shared memory: a CTA finds room beside one
// of the main kernel, and is there when that leaves.)
constexpr int kJoinThreads = 128;
constexpr int kJoinRows = 16;

__global__ void __launch_bounds__(kJoinThreads, 16) chunk_join_kernel(const ChunkParams p, int grid) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int cta = blockIdx.x;
    wait_prior_grid();
    allow_dependent_launch();
    // the pieces behind the first are the first ones of the CTAs behind (of those that have
    // one), up to the one that ends the block
    auto flags_of = [&](int c) { return c < grid ? __ldcg(&p.slots[2 * c + (c == cta)].w) : 0; };
    const int4 head = __ldcg(p.slots + 2 * cta + 1);
    const int flags = flags_of(cta + lane);
    const int rows = head.z * p.G;
    if (!(head.w & kUsed) || (int)blockIdx.y * kJoinRows >= rows) return;
    int last = cta;            // the CTA with the block's end
    for (int c = cta; last == cta && c < grid; c += 32) {
        const unsigned ends = __ballot_sync(0xffffffffu, (c == cta ? flags : flags_of(c + lane)) & kEnds);
        if (ends) last = c + __ffs(ends) - 1;
    }
    if (last == cta) return;   // (a wait gave up; the status says so)
    for (int r = blockIdx.y * kJoinRows + warp; r < min(rows, ((int)blockIdx.y + 1) * kJoinRows); r += kJoinThreads / 32) {
        float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
        float top = kNegInf, total = 0.f;
        for (int c = cta; c <= last; c += 32) {
            const int used = c + lane <= last ? (c == cta ? flags : flags_of(c + lane)) & kUsed : 0;
            const float2 ml = used ? __ldcg(p.part_ml + (size_t)(2 * (c + lane) + (c + lane == cta)) * p.rows + r)
                                   : make_float2(kNegInf, 0.f);
            float most = ml.x;
#pragma unroll
            for (int d = 16; d > 0; d /= 2) most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, d));
            most = fmaxf(most, top);
            // (no score of these is a number, or there is none; NaN scores leave a NaN sum and
            // outputs, which are the result)
            if (most == kNegInf && !__any_sync(0xffffffffu, ml.y != 0.f)) continue;
            // (outputs are divided by their sums already)
            float w = ml.y * ex2(ml.x - most), sum = w;
#pragma unroll
            for (int d = 16; d > 0; d /= 2) sum += __shfl_xor_sync(0xffffffffu, sum, d);
            float f = total * ex2(top - most);
            sum += f;
            const float inv = sum > 0.f ? rcp(sum) : 0.f;
            f *= inv;
            w *= inv;
            o = make_float4(o.x * f, o.y * f, o.z * f, o.w * f);
            unsigned left = __ballot_sync(0xffffffffu, used);
            while (left) {
                float4 x[4];
                float g[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const int at = left ? __ffs(left) - 1 : 0;
                    g[k] = __shfl_sync(0xffffffffu, w, at);
                    x[k] = make_float4(0.f, 0.f, 0.f, 0.f);
                    if (left)
                        x[k] = __ldcg(reinterpret_cast<const float4*>(
                                          p.part_o + ((size_t)(2 * (c + at) + (c + at == cta)) * p.rows + r) * kD) + lane);
                    else
                        g[k] = 0.f;
                    left &= left - 1;
                }
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    o.x = fmaf(x[k].x, g[k], o.x);
                    o.y = fmaf(x[k].y, g[k], o.y);
                    o.z = fmaf(x[k].z, g[k], o.z);
                    o.w = fmaf(x[k].w, g[k], o.w);
                }
            }
            top = most;
            total = sum;
        }
        uint2* dst = reinterpret_cast<uint2*>(
            p.out + ((size_t)(head.x + r / p.G) * p.Hq + (size_t)head.y * p.G + r % p.G) * kD);
        dst[lane] = make_uint2(pack_bf16x2(o.x, o.y), pack_bf16x2(o.z, o.w));
    }
}

// ------------------------------------------------------------------ the host
PFN_cuTensorMapEncodeTiled_v12000 encoder() {
    static std::atomic<PFN_cuTensorMapEncodeTiled_v12000> fn{nullptr};
    if (!fn) {
        void* ptr = nullptr;
        cudaDriverEntryPointQueryResult q;
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &ptr, 12000, cudaEnableDefault, &q) == cudaSuccess &&
            q == cudaDriverEntryPointSuccess)
            fn = reinterpret_cast<PFN_cuTensorMapEncodeTiled_v12000>(ptr);
    }
    return fn;
}

cs_status encode(CUtensorMap* map, const void* data, int rank, const cuuint64_t* dims, const cuuint64_t* strides,
                 const cuuint32_t* box) {
    auto enc = encoder();
    if (!enc) return fail(CS_ERR_CUDA, "cuTensorMapEncodeTiled is not available from the driver");
    const cuuint32_t ones[5] = {1, 1, 1, 1, 1};
    const CUresult r = enc(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, rank, const_cast<void*>(data), dims, strides, box, ones,
                           CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                           CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    return r == CUDA_SUCCESS ? CS_OK : fail(CS_ERR_CUDA, "cuTensorMapEncodeTiled failed (CUresult %d)", (int)r);
}

// A pool as 8-key groups (64 dims, 8 keys, 2 dim halves, groups), so that a box of a
// page's keys lands as [group][half][8 keys][64 dims]
cs_status encode_pool(CUtensorMap* map, const void* pool, const cs_attn_dims& d) {
    const cuuint64_t dims[4] = {64, 8, 2, (cuuint64_t)d.num_pages * d.n_kv_heads * (d.page_size / 8)};
    const cuuint64_t strides[3] = {256, 128, 2048};
    const cuuint32_t box[4] = {64, 8, 2, (cuuint32_t)(d.page_size < kKeys ? d.page_size : kKeys) / 8};
    return encode(map, pool, 4, dims, strides, box);
}

// Query rows of one KV head of some tokens, a dim half at a time: [token][head][64 dims]
cs_status encode_rows(CUtensorMap* map, const void* q, const cs_attn_dims& d, int tokens, int64_t stride, int box_tokens) {
    const cuuint64_t dims[3] = {kD, (cuuint64_t)d.n_q_heads, (cuuint64_t)tokens};
    const cuuint64_t strides[2] = {kD * 2, (cuuint64_t)stride * 2};
    const cuuint32_t box[3] = {64, (cuuint32_t)(d.n_q_heads / d.n_kv_heads), (cuuint32_t)box_tokens};
    return encode(map, q, 3, dims, strides, box);
}

struct Layout {
    int rows;
    size_t done, slots, ml, o, bytes;
};
size_t align_up(size_t x) { return (x + 255) / 256 * 256; }
Layout layout(const cs_attn_dims& d, int tokens, int grid) {
    Layout l;
    const long long all = (long long)tokens * (d.n_q_heads / d.n_kv_heads);
    l.rows = all < kRows ? ((int)all + 15) / 16 * 16 : kRows;   // (a warp's, whole)
    l.done = 256;
    l.slots = align_up(l.done + sizeof(int) * grid);
    l.ml = align_up(l.slots + sizeof(int4) * 2 * grid);
    l.o = align_up(l.ml + sizeof(float2) * 2 * grid * l.rows);
    l.bytes = align_up(l.o + sizeof(float) * kD * 2 * grid * l.rows);
    return l;
}

}  // namespace

size_t chunk_attention_workspace_bytes(const cs_attn_dims& d, int tokens, int sm_count) {
    return layout(d, tokens, sm_count).bytes;
}

cs_status launch_chunk_attention(const cs_attn_dims& d, const void* q, int64_t q_stride, int tokens,
                                 const void* k_pages, const void* v_pages, const int32_t* page_table,
                                 const int32_t* ctx_lens, const int32_t* q_starts, void* out, void* workspace,
                                 cudaStream_t stream) {
    const int grid = current_sm_count();
    const Layout l = layout(d, tokens, grid);
    uint8_t* ws = static_cast<uint8_t*>(workspace);
    ChunkParams p{};
    p.batch = RaggedBatch{ctx_lens, q_starts, d.batch, tokens, q_starts ? 0 : tokens / d.batch,
                          d.max_pages_per_seq * d.page_size};
    p.page_table = page_table;
    p.out = static_cast<__nv_bfloat16*>(out);
    p.status = reinterpret_cast<int*>(ws);
    p.done = reinterpret_cast<int*>(ws + l.done);
    p.slots = reinterpret_cast<int4*>(ws + l.slots);
    p.part_ml = reinterpret_cast<float2*>(ws + l.ml);
    p.part_o = reinterpret_cast<float*>(ws + l.o);
    p.Hq = d.n_q_heads;
    p.Hkv = d.n_kv_heads;
    p.G = d.n_q_heads / d.n_kv_heads;
    p.ps = d.page_size;
    while ((1 << p.ps_log2) < d.page_size) ++p.ps_log2;
    p.max_pages = d.max_pages_per_seq;
    p.P = d.num_pages;
    p.block_tokens = kRows / p.G;
    p.by_block = HostDivisor::of((uint32_t)p.block_tokens);
    p.by_grid = HostDivisor::of((uint32_t)grid);
    p.small_tokens = p.G < kSmallQRows ? kSmallQRows / p.G : 1;
    p.rows = l.rows;
    p.scale_log2 = (d.sm_scale > 0.f ? d.sm_scale : 1.0f / sqrtf((float)kD)) * 1.4426950408889634f;

    CUtensorMap mk, mv, mq, ms;
    cs_status st = encode_pool(&mk, k_pages, d);
    if (st == CS_OK) st = encode_pool(&mv, v_pages, d);
    if (st == CS_OK) st = encode_rows(&mq, q, d, tokens, q_stride, p.block_tokens);
    if (st == CS_OK) st = encode_rows(&ms, q, d, tokens, q_stride, p.small_tokens);
    if (st != CS_OK) return st;
    // whether the weight of all blocks is sure to fit 32 bits
    const long long most_blocks = (tokens + p.block_tokens - 1) / p.block_tokens + (long long)d.batch;
    const bool wide = (p.batch.max_keys + (long long)kBeginKeys) * p.Hkv > 0x7fffffffLL / most_blocks;
    const bool wide_out = reinterpret_cast<uintptr_t>(out) % 32 == 0;
    auto kern = wide_out ? (wide ? chunk_attention_kernel<uint64_t, true> : chunk_attention_kernel<uint32_t, true>)
                         : (wide ? chunk_attention_kernel<uint64_t, false> : chunk_attention_kernel<uint32_t, false>);
    {
        static std::atomic<bool> done[4][64];
        const int which = 2 * wide_out + wide;
        int dev = 0;
        cudaError_t e = cudaGetDevice(&dev);
        if (e != cudaSuccess) return cuda_fail(e, "cudaGetDevice");
        if (dev < 0 || dev >= 64 || !done[which][dev]) {
            e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmem);
            if (e != cudaSuccess) return cuda_fail(e, "cudaFuncSetAttribute(chunk_attention_kernel)");
            if (dev >= 0 && dev < 64) done[which][dev] = true;
        }
    }
    // As many blocks as there may be (the lengths are the device's): with few of them each
    // has many pieces, and joining them is work for the whole card.
    const long long by_tokens = (tokens + p.block_tokens - 1) / p.block_tokens;
    // (Nor is there anything to join where no context is long enough for a cut.)
    const bool uncut = p.batch.max_keys <= kUncut;
    p.cut_back = uncut ? 1 << 30 : kCutBack;
    p.join_here = uncut || kJoinBlocks * p.Hkv * (by_tokens > d.batch ? by_tokens : d.batch < tokens ? d.batch : tokens) >= grid;
    if (!p.join_here) p.rows = (int)std::min((long long)kRows, (long long)tokens * p.G);
    p.least = p.join_here ? 0 : kLeast + kLeastRow * p.rows;
    for (p.b0 = 0; p.b0 < d.batch; p.b0 += kMaxBatch) {
        p.nb = d.batch - p.b0 < kMaxBatch ? d.batch - p.b0 : kMaxBatch;
        cudaError_t e = launch_dependent(kern, dim3(grid), dim3(kThreads), (size_t)kSmem, stream, mk, mv,
                                         mq, ms, p);
        if (e != cudaSuccess) return cuda_fail(e, "chunk_attention_kernel launch");
        if (p.join_here) continue;
        e = launch_dependent(chunk_join_kernel, dim3(grid, (l.rows + kJoinRows - 1) / kJoinRows), dim3(kJoinThreads), 0, stream,
                             p, grid);
        if (e != cudaSuccess) return cuda_fail(e, "chunk_join_kernel launch");
    }
    return CS_OK;
}

}  // namespace cs
