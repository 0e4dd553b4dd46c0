// logprobs.cu -- log probabilities of given tokens, the entropy and the top
// alternatives of their rows (cs_logprobs), in one pass over the logits.
//
// A cluster of 1 to 8 CTAs takes a row, each a contiguous slice in tiles of
// kTile 16-byte vectors (rows of any alignment are read in 16-byte blocks of
// memory, what lies outside the row counts as -inf).  A thread keeps a running
// maximum m, and with it S = sum w and U = sum w d of the weights
// w = 2^(d log2(e) / T), d = z - m; so
//     ln sum exp(z / T) = m / T + ln S,   H = ln S - U / (S T).
//
// The alternatives: a logit and its id are one ordered number (the larger
// logit, then the lower id).  While it streams, a thread keeps the maximum of
// each sixteenth of its logits (a cell) in shared memory.  At the end the n-th
// largest of the threads' maxima is a bound that at least n logits reach, and
// few more do (n = 20 of 128256: 21 on average): the cells that reach it are
// read again, from L2, and their keys ranked.  Rows on which too many cells or
// keys reach the bound (ties by the thousand, rows made to that end) are read
// again tile by tile, with a list that is cut to the n best and a bound that
// grows.  Keys are unique, so the order in which they arrive changes nothing.
// The first CTA of the cluster merges the slices' sums and keys through
// distributed shared memory.
//
// What bounds it: many rows the instructions of a logit (conversion, maximum,
// exponential, two sums, the cell's maximum; issue 65% busy) and the last wave: 608
// CTAs are resident, and 608 wanted rows of 128256 bf16 logits with 20 alternatives
// take 35 us, 616 45, 1216 65 and 1276 (two waves and 60 rows) 76, 4.3 TB/s (61 without
// alternatives).  A row alone is a chain of latencies: 32001 fp32 logits 8 us
// with the call's host part.
#include "cs_internal.h"
#include "cs_device.cuh"

namespace cs {
namespace {

constexpr int kThreads = 256;
constexpr int kVecs = 4;                       // 16-byte vectors of a thread's tile
constexpr int kTile = kThreads * kVecs;
constexpr int kMaxCluster = 8;
constexpr int kListFull = 2 * CS_MAX_TOP + 24;  // a list of 2 n + 24 keys is cut to the n best
constexpr int kCells = 16;                     // parts of a thread's logits
constexpr int kMaxCells = 512;                 // of the CTA's cells that are read again
constexpr int kSlack = 8;                      // more keys than n that a bound may let through
constexpr int kList = 2048;                    // what the list takes
static_assert(kList >= kListFull + (CS_MAX_TOP + kSlack) * kVecs * 8, "a tile's keys above its threads' n-th best fit");
static_assert(kListFull <= kThreads && kMaxCluster * CS_MAX_TOP <= kThreads, "a thread a key");

using Key = unsigned long long;

struct LogprobParams {
    const void* logits;
    const int32_t* tokens;
    float* logprob;
    float* entropy;
    int32_t* top_tokens;
    float* top_logprobs;
    int V, n_top;
    long long stride;
    float c;                     // log2(e) / T
    float i_hi, i_lo;            // 1 / T
    float d_min;                 // weights of logits further below the maximum are 0
};

// Larger logit, then lower id (-0 is 0).
__device__ __forceinline__ Key key_of(float z, int v) {
    const uint32_t b = __float_as_uint(z + 0.f);
    return (Key)(b & 0x80000000u ? ~b : b | 0x80000000u) << 32 | (uint32_t)~v;
}
__device__ __forceinline__ float logit_of(Key k) {
    const uint32_t b = (uint32_t)(k >> 32);
    return __uint_as_float(b & 0x80000000u ? b & 0x7fffffffu : ~b);
}
__device__ __forceinline__ int id_of(Key k) { return (int)~(uint32_t)k; }

__device__ __forceinline__ uint32_t cluster_rank() {
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ void cluster_sync() {
    asm volatile("barrier.cluster.arrive.aligned;\n\tbarrier.cluster.wait.aligned;" ::: "memory");
}
// the same shared-memory word of CTA `rank` of the cluster
__device__ __forceinline__ uint32_t at_rank(const void* p, uint32_t rank) {
    uint32_t a;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(smem_u32(p)), "r"(rank));
    return a;
}
__device__ __forceinline__ Key load_key(uint32_t a) {
    Key k;
    asm volatile("ld.shared::cluster.u64 %0, [%1];" : "=l"(k) : "r"(a) : "memory");
    return k;
}
__device__ __forceinline__ float load_float(uint32_t a) {
    float f;
    asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(f) : "r"(a) : "memory");
    return f;
}

struct Sums {
    float m, S, U;
};
// Sums of two sets of weights under the larger of their maxima.
__device__ __forceinline__ Sums join(const Sums& a, const Sums& b, float c, float d_min) {
    Sums r;
    r.m = fmaxf(a.m, b.m);
    if (r.m == kNegInf) return a;
    const float da = fmaxf(a.m - r.m, d_min), db = fmaxf(b.m - r.m, d_min);
    const float wa = ex2(da * c), wb = ex2(db * c);
    r.S = a.S * wa + b.S * wb;
    r.U = wa * fmaf(a.S, da, a.U) + wb * fmaf(b.S, db, b.U);
    return r;
}

template <bool kF32>
__device__ __forceinline__ float element(const uint4& v, int i) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
    if constexpr (kF32) return __uint_as_float(w[i]);
    else return __uint_as_float(i & 1 ? w[i / 2] & 0xffff0000u : w[i / 2] << 16);
}

__device__ __forceinline__ uint32_t max_bf16x2(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("max.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}

template <bool kF32, bool kTop>
__global__ void __launch_bounds__(kThreads, 4) logprobs_kernel(const LogprobParams p) {
    constexpr int kPer = kF32 ? 4 : 8;          // logits of a vector
    __shared__ Key s_list[kTop ? kList : 1];
    __shared__ Key s_best[kTop ? kThreads : 1];
    __shared__ float s_cell[kTop ? kCells : 1][kTop ? kThreads : 1];
    __shared__ int s_cells[kTop ? kMaxCells : 1];
    __shared__ int s_cell_count;
    __shared__ Key s_kept[kTop ? CS_MAX_TOP * (kList / kThreads) : 1];
    __shared__ int s_kept_count;
    __shared__ Key s_top[CS_MAX_TOP];           // the slice's best, in order
    __shared__ Key s_bound;
    __shared__ int s_count;
    __shared__ Sums s_sums[kThreads / 32];
    __shared__ Sums s_slice;

    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    uint32_t ranks;
    asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(ranks));
    const uint32_t rank = cluster_rank();
    const int r = blockIdx.x / ranks, n = p.n_top, full_at = 2 * n + 24;
    wait_prior_grid();
    allow_dependent_launch();
    const int tok = __ldcg(p.tokens + r);
    if (tok < 0) {   // (the whole cluster leaves)
        if (rank == 0) {
            if (tid == 0) {
                p.logprob[r] = kNegInf;
                if (p.entropy) p.entropy[r] = 0.f;
            }
            if (tid < n) {
                p.top_tokens[(size_t)r * n + tid] = -1;
                p.top_logprobs[(size_t)r * n + tid] = kNegInf;
            }
        }
        return;
    }
    const char* row = static_cast<const char*>(p.logits) + (size_t)r * p.stride * (kF32 ? 4 : 2);
    // the row in 16-byte blocks of memory: logit 0 is number `skip` of the first one
    const uint4* blocks = reinterpret_cast<const uint4*>(reinterpret_cast<uintptr_t>(row) & ~uintptr_t(15));
    const int skip = (int)((reinterpret_cast<uintptr_t>(row) & 15) / (kF32 ? 4 : 2));
    const int n_blocks = (skip + p.V + kPer - 1) / kPer;
    const int per = ((n_blocks + ranks - 1) / ranks + 31) / 32 * 32;     // whole 512-byte pieces a slice
    const int first = min((int)rank * per, n_blocks), last = min(first + per, n_blocks);
    float z_tok = 0.f;
    if (rank == 0 && tid == 0 && tok < p.V)
        z_tok = kF32 ? __ldcg(reinterpret_cast<const float*>(row) + tok)
                     : bf16_bits_to_float(__ldcg(reinterpret_cast<const uint16_t*>(row) + tok));
    if (kTop && tid == 0) {
        s_bound = 0;
        s_count = 0;
        s_cell_count = 0;
    }

    constexpr uint32_t kNone = kF32 ? 0xff800000u : 0xff80ff80u;        // -inf
    auto load = [&](int base, uint4 (&v)[kVecs]) {
#pragma unroll
        for (int u = 0; u < kVecs; ++u) {
            const int b = base + u * kThreads + tid;
            v[u] = b < last ? __ldcg(blocks + b) : make_uint4(kNone, kNone, kNone, kNone);
        }
    };
    // -inf for what a row's first and last block hold of others
    auto trim_vector = [&](int b, uint4& x) {
        if ((b != 0 || skip == 0) && (b + 1 != n_blocks || (b + 1) * kPer - skip == p.V)) return;
        uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            const int id = b * kPer - skip + i;
            if (id >= 0 && id < p.V) continue;
            if (kF32) w[i & 3] = kNone;
            else if (i & 1) w[i / 2] = (w[i / 2] & 0xffffu) | 0xff800000u;
            else w[i / 2] = (w[i / 2] & 0xffff0000u) | 0xff80u;
        }
        x = make_uint4(w[0], w[1], w[2], w[3]);
    };
    auto trim = [&](int base, uint4 (&v)[kVecs]) {
#pragma unroll
        for (int u = 0; u < kVecs; ++u) {
            const int b = base + u * kThreads + tid;
            if (b < last) trim_vector(b, v[u]);
        }
    };
    auto place = [&](Key k, const Key* keys, int count) {   // how many of the keys are larger
        int at = 0;
#pragma unroll 4
        for (int j = 0; j < count; ++j) at += keys[j] > k;
        return at;
    };
    // The largest T for which n or more of the threads' numbers reach T (0 where
    // fewer than n are not 0), or one that n + kSlack do at most; and how many do.
    auto nth_of = [&](uint32_t o, int& reach) {
        uint32_t T = 0;
        reach = kThreads;
        for (int bit = 31; bit >= (kF32 ? 0 : 16); --bit) {   // (a bf16's low half is 0, or all ones)
            const int c = __syncthreads_count(o >= (T | 1u << bit));
            if (c < n) continue;
            T |= 1u << bit;
            reach = c;
            if (c <= n + kSlack) break;
        }
        return T;
    };
    // Cuts the list; the bound follows.  `last_cut`: to the n best, in order in
    // s_top; else to as many as reach the n-th best logit (or a few more).  Between barriers.
    auto cut = [&](bool last_cut) {
        int count = min(s_count, kList);
        Key mine = 0;
        if (count > kThreads) {
            // the n best lie with the threads whose own best is among the n best of those
            for (int j = tid; j < count; j += kThreads) mine = s_list[j] > mine ? s_list[j] : mine;
            s_best[tid] = mine;
            __syncthreads();
            const bool in = mine != 0 && place(mine, s_best, kThreads) < n;
            if (tid == 0) s_kept_count = 0;
            __syncthreads();
            if (in)
                for (int j = tid; j < count; j += kThreads) s_kept[atomicAdd(&s_kept_count, 1)] = s_list[j];
            __syncthreads();
            count = s_kept_count;
            mine = tid < count ? s_kept[tid] : 0;
            __syncthreads();
        } else {
            mine = tid < count ? s_list[tid] : 0;
        }
        int reach = count;
        uint32_t T = 0;
        if (count > n) T = nth_of((uint32_t)(mine >> 32), reach);
        if (tid == 0) s_kept_count = 0;
        __syncthreads();   // (and s_list, s_kept are read)
        const bool keep = mine != 0 && (uint32_t)(mine >> 32) >= T;
        if (last_cut || reach > n + kSlack) {   // (many equal logits: by their ids)
            if (keep) s_best[atomicAdd(&s_kept_count, 1)] = mine;
            if (tid < n) s_top[tid] = 0;
            __syncthreads();
            count = s_kept_count;
            mine = tid < count ? s_best[tid] : 0;
            const int at = mine ? place(mine, s_best, count) : n;
            if (at < n) s_top[at] = mine;
            __syncthreads();
            if (tid < n) s_list[tid] = s_top[tid];
            if (tid == 0) {
                s_count = min(count, n);
                if (s_top[n - 1] > s_bound) s_bound = s_top[n - 1];
            }
        } else {
            if (keep) s_list[atomicAdd(&s_kept_count, 1)] = mine;
            if (tid == 0) {
                s_count = reach;
                const Key bound = T ? ((Key)T << 32) - 1 : 0;
                if (bound > s_bound) s_bound = bound;
            }
        }
        __syncthreads();
    };

    auto top_of = [&](const uint4& x) {   // a vector's largest logit
        if constexpr (kF32) {
            return fmaxf(fmaxf(element<true>(x, 0), element<true>(x, 1)), fmaxf(element<true>(x, 2), element<true>(x, 3)));
        } else {
            const uint32_t m2 = max_bf16x2(max_bf16x2(x.x, x.y), max_bf16x2(x.z, x.w));
            return fmaxf(__uint_as_float(m2 << 16), __uint_as_float(m2 & 0xffff0000u));
        }
    };
    auto append = [&](Key k) {   // whether the list is to be cut
        const int at = atomicAdd(&s_count, 1);
        if (at < kList) s_list[at] = k;
        return at + 1 >= full_at;
    };
    // the keys of a vector that reach `least` and lie above the bound, in a rolled
    // loop: little code for few threads
    auto push_vector = [&](uint4 w, int id, float least, Key bound) {
        bool full = false;
#pragma unroll 1
        for (int i = 0; i < kPer; ++i) {
            const float z = element<kF32>(w, 0);
            if (kF32) {
                w.x = w.y;
                w.y = w.z;
                w.z = w.w;
            } else {
                w.x = __byte_perm(w.x, w.y, 0x5432);
                w.y = __byte_perm(w.y, w.z, 0x5432);
                w.z = __byte_perm(w.z, w.w, 0x5432);
                w.w >>= 16;
            }
            if (z < least || z == kNegInf) continue;
            const Key k = key_of(z, id + i);
            if (k > bound) full |= append(k);
        }
        return full;
    };

    Sums t{kNegInf, 0.f, 0.f};
    uint4 v[kVecs], ahead[kVecs];
    const int tiles = (last - first + kTile - 1) / kTile, cell_tiles = (tiles + kCells - 1) / kCells;
    int cell = 0, in_cell = 0;
    float cell_top = kNegInf;
    load(first, v);
    for (int base = first; base < last; base += kTile) {
        load(base + kTile, ahead);
        if ((base == 0 && skip > 0) || base + kTile >= n_blocks) trim(base, v);
        // ---- the tile's maximum and sums
        float top;
        if constexpr (kF32) {
            top = kNegInf;
#pragma unroll
            for (int u = 0; u < kVecs; ++u)
#pragma unroll
                for (int i = 0; i < 4; ++i) top = fmaxf(top, element<true>(v[u], i));
        } else {
            uint32_t t2 = kNone;
#pragma unroll
            for (int u = 0; u < kVecs; ++u)
                t2 = max_bf16x2(t2, max_bf16x2(max_bf16x2(v[u].x, v[u].y), max_bf16x2(v[u].z, v[u].w)));
            top = fmaxf(__uint_as_float(t2 << 16), __uint_as_float(t2 & 0xffff0000u));
        }
        if (top > t.m) {
            const float d = fmaxf(t.m - top, p.d_min), w = ex2(d * p.c);
            t.U = w * fmaf(t.S, d, t.U);
            t.S *= w;
            t.m = top;
        }
        if (top > kNegInf) {
            const uint64_t m2 = f2_pack(t.m, t.m), c2 = f2_pack(p.c, p.c);
            uint64_t S2 = 0, U2 = 0;
#pragma unroll
            for (int u = 0; u < kVecs; ++u)
#pragma unroll
                for (int i = 0; i < kPer; i += 2) {
                    float d0, d1, w0, w1;
                    f2_unpack(f2_sub(f2_pack(element<kF32>(v[u], i), element<kF32>(v[u], i + 1)), m2), d0, d1);
                    const uint64_t d2 = f2_pack(fmaxf(d0, p.d_min), fmaxf(d1, p.d_min));   // (a -inf too)
                    f2_unpack(f2_mul(d2, c2), w0, w1);
                    const uint64_t w2 = f2_pack(ex2(w0), ex2(w1));
                    S2 = f2_add(S2, w2);
                    U2 = f2_fma(w2, d2, U2);
                }
            float S0, S1, U0, U1;
            f2_unpack(S2, S0, S1);
            f2_unpack(U2, U0, U1);
            t.S += S0 + S1;
            t.U += U0 + U1;
        }
        if constexpr (kTop) {
            cell_top = fmaxf(cell_top, top);
            if (++in_cell == cell_tiles || base + kTile >= last) {
                s_cell[cell++][tid] = cell_top;
                cell_top = kNegInf;
                in_cell = 0;
            }
        }
#pragma unroll
        for (int u = 0; u < kVecs; ++u) v[u] = ahead[u];
    }

    if constexpr (kTop) {
        __syncthreads();   // (the counts of 0)
        const uint32_t mine = t.m == kNegInf ? 0 : (uint32_t)(key_of(t.m, 0) >> 32);
        int reach;
        const uint32_t T = nth_of(mine, reach);
        const float least = T ? logit_of((Key)T << 32) : -3.4028235e38f;   // (fewer than n threads have any: all of theirs)
        if (t.m >= least)
            for (int j = 0; j < cell; ++j)
                if (s_cell[j][tid] >= least) {
                    const int at = atomicAdd(&s_cell_count, 1);
                    if (at < kMaxCells) s_cells[at] = j * kThreads + tid;
                }
        __syncthreads();
        const int cells = s_cell_count, cell_vecs = cell_tiles * kVecs;
        if (cells <= kMaxCells) {
            for (int j = tid; j < cells * cell_vecs; j += kThreads) {
                const int of = s_cells[j / cell_vecs], k = j % cell_vecs;   // vector k of the cell
                const int b = first + (of / kThreads * cell_vecs + k) * kThreads + of % kThreads;
                if (b >= last) continue;
                uint4 x[kVecs] = {__ldcg(blocks + b)};
                trim_vector(b, x[0]);
                if (top_of(x[0]) >= least) push_vector(x[0], b * kPer - skip, least, 0);
            }
        }
        __syncthreads();
        if (cells > kMaxCells || s_count > kList) {
            __syncthreads();
            if (tid == 0) s_count = 0;
            __syncthreads();
            for (int base = first; base < last; base += kTile) {
                load(base, v);
                if ((base == 0 && skip > 0) || base + kTile >= n_blocks) trim(base, v);
                const int id0 = base * kPer - skip;   // the tile's first id
                auto id_at = [&](int u) { return id0 + (u * kThreads + tid) * kPer; };
                auto push = [&]() {
                    const Key bound = s_bound;
                    const float at_least = bound ? logit_of(bound) : kNegInf;
                    bool full = false;
#pragma unroll
                    for (int u = 0; u < kVecs; ++u)
                        if (top_of(v[u]) >= at_least) full |= push_vector(v[u], id_at(u), at_least, bound);
                    return full;
                };
                const bool begin = base == first;
                if (!begin && !__syncthreads_or(push())) continue;
                if (begin || s_count > kList) {
                    // a bound from this tile alone, under which the list takes it (again);
                    // what lies in the list from the tiles before came first
                    Key best = 0, kept = tid < min(s_count, kListFull) ? s_list[tid] : 0;
                    if (kept && id_of(kept) >= id0) kept = 0;
#pragma unroll
                    for (int u = 0; u < kVecs; ++u)
#pragma unroll
                        for (int i = 0; i < kPer; ++i) {
                            const float z = element<kF32>(v[u], i);
                            const Key k = z == kNegInf ? 0 : key_of(z, id_at(u) + i);
                            best = k > best ? k : best;
                        }
                    s_best[tid] = best;
                    __syncthreads();
                    if (tid == 0) s_count = 0;
                    if (best > s_bound && place(best, s_best, kThreads) == n - 1) s_bound = best - 1;   // (one thread's)
                    __syncthreads();
                    if (kept) append(kept);
                    push();
                    __syncthreads();
                }
                cut(false);
            }
        }
    }

    // ---- the slice's sums and best keys
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) {
        const Sums o{__shfl_xor_sync(0xffffffffu, t.m, off), __shfl_xor_sync(0xffffffffu, t.S, off),
                     __shfl_xor_sync(0xffffffffu, t.U, off)};
        t = join(t, o, p.c, p.d_min);
    }
    if (lane == 0) s_sums[warp] = t;
    __syncthreads();
    if (kTop) cut(true);
    if (tid == 0) {
        for (int w = 1; w < kThreads / 32; ++w) t = join(t, s_sums[w], p.c, p.d_min);
        s_slice = t;
    }
    if (ranks > 1) {
        cluster_sync();
        if (rank == 0 && tid == 0) {
            for (uint32_t k = 1; k < ranks; ++k) {
                const Sums o{load_float(at_rank(&s_slice.m, k)), load_float(at_rank(&s_slice.S, k)),
                             load_float(at_rank(&s_slice.U, k))};
                t = join(t, o, p.c, p.d_min);
            }
            s_sums[0] = t;
        }
        if (kTop && rank == 0) {
            const int count = (int)ranks * n;
            Key mine = 0;
            if (tid < count) mine = load_key(at_rank(&s_top[tid % n], tid / n));
            s_best[tid] = mine;
            __syncthreads();
            const int at = mine ? place(mine, s_best, count) : n;
            __syncthreads();   // (its own s_top is read above)
            if (tid < n) s_top[tid] = 0;
            __syncthreads();
            if (at < n) s_top[at] = mine;
        }
        cluster_sync();
        if (rank != 0) return;
    } else if (tid == 0) {
        s_sums[0] = t;
    }
    __syncthreads();
    const Sums all = s_sums[0];
    const float lse = lg2(all.S) * kLn2;
    auto lp = [&](float z) {
        const float d = z - all.m;   // (-inf where the difference, or d / T, passes fp32)
        return all.m == kNegInf || d * p.i_hi == kNegInf ? kNegInf : fmaf(d, p.i_hi, fmaf(d, p.i_lo, -lse));
    };
    if (tid == 0) {
        p.logprob[r] = tok < p.V ? lp(z_tok) : kNegInf;
        if (p.entropy) p.entropy[r] = all.m == kNegInf ? 0.f : fmaxf(0.f, lse - all.U / all.S * p.i_hi);
    }
    if (kTop && tid < n) {
        const Key k = s_top[tid];
        p.top_tokens[(size_t)r * n + tid] = k ? id_of(k) : -1;
        p.top_logprobs[(size_t)r * n + tid] = k ? lp(logit_of(k)) : kNegInf;
    }
}

// CTAs a row: more than one only while all of them have an SM of their own and
// some 16 KB each.  48 rows of 128256 bf16 logits: 15.5, 12.5, 13.1 and 15.1 us
// with 1, 2, 4 and 8; one row 14.5, 11.6, 11.1, 11.3; 160 rows 18.7, 20.4, 21.3, 30.3.
int cluster_of(const cs_logprob_dims& d) {
    const size_t bytes = (size_t)d.vocab * (d.logit_dtype == CS_F32 ? 4 : 2);
    int c = 1;
    while (c < kMaxCluster && (long long)d.rows * 2 * c <= current_sm_count() && bytes / (2 * c) >= 16384) c *= 2;
    return c;
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
    const double i = 1.0 / (double)temperature, c = 1.4426950408889634073599 * i;
    p.c = (float)c;
    p.i_hi = (float)i;
    p.i_lo = (float)(i - (double)p.i_hi);
    p.d_min = (float)(-300.0 / c);
    using Kern = void (*)(const LogprobParams);
    static const Kern kerns[2][2] = {{logprobs_kernel<false, false>, logprobs_kernel<false, true>},
                                     {logprobs_kernel<true, false>, logprobs_kernel<true, true>}};
    const int cluster = cluster_of(d);
    if ((long long)d.rows * cluster > 0x7fffffffLL) return fail(CS_ERR_UNSUPPORTED, "too many rows in one call");
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = cluster;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(d.rows * cluster));
    cfg.blockDim = dim3(kThreads);
    cfg.stream = stream;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    const cudaError_t e = cudaLaunchKernelEx(&cfg, kerns[d.logit_dtype == CS_F32][d.n_top > 0], p);
    return e == cudaSuccess ? CS_OK : cuda_fail(e, "logprobs_kernel launch");
}

}  // namespace cs
