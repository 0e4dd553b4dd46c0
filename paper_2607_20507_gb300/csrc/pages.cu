// pages.cu -- pages of a cache that rows of the page table share, give back and
// that move together (cs_kv_fork, cs_kv_release, cs_kv_compact; the copies of a fork
// or a compaction in more pools than one call takes: cs_kv_fork_more,
// cs_kv_compact_more).
//
// The counts alone say which pages are free, so there is no list to keep: a
// fork takes the lowest free ids, found by a scan of the counts.  Every result
// is a function of the inputs: places come from prefix sums, and the only
// atomics are additions to whole numbers.
//
// What bounds them: a fork and a release are chains of a few dependent loads
// and the launches (a release and a fork of 4 rows 10 us, of 192 rows 16); a
// compaction reads the counts twice and the table once and then copies pages at
// the memory's rate: 26,637 pages of 18 KB take 178 us, 5.5 TB/s; 239 of 64 KB,
// 20.5 us, two launches and 16 MB each way.
#include "cs_internal.h"
#include "cs_device.cuh"

namespace cs {
namespace {

constexpr int kPiece = 128;             // 16-byte vectors that a warp copies at a time, four a lane in flight

struct PagePools {
    uint4* data[CS_MAX_PAGE_POOLS];
    uint32_t vecs[CS_MAX_PAGE_POOLS];   // 16-byte vectors of a page
    uint32_t first[CS_MAX_PAGE_POOLS];  // a page's pieces in the pools before
    uint32_t pieces;                    // and in all
    int n;
};

struct PageParams {
    int32_t* table;      // [R, max_pages]
    int32_t* lens;       // [R]
    int32_t* refs;       // [P]
    int R, max_pages, ps, P;
};

__device__ __forceinline__ int clamped_len(const PageParams& p, int L) {
    return max(0, min(L, p.max_pages * p.ps));
}

// Sum over the block's threads before this one, and the block's total.
template <int kThreads, class T>
__device__ __forceinline__ T block_scan(T v, T* s_warp, T& total) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    T inc = v;
#pragma unroll
    for (int off = 1; off < 32; off <<= 1) {
        const T y = __shfl_up_sync(0xffffffffu, inc, off);
        if (lane >= off) inc += y;
    }
    __syncthreads();   // (s_warp of the scan before)
    if (lane == 31) s_warp[warp] = inc;
    __syncthreads();
    T before = 0, all = 0;
    for (int w = 0; w < kThreads / 32; ++w) {
        const T x = s_warp[w];
        if (w < warp) before += x;
        all += x;
    }
    total = all;
    return before + inc - v;
}

// Of the 16 pages from base + 16 threadIdx.x on, which have a count of 0 (kFree) or
// another (else): a bit each.  A warp reads its 512 counts 32 at a time (a thread its
// own 16 would touch every sector eight times); all of it takes part.
constexpr int kPer = 16;
template <bool kFree>
__device__ __forceinline__ uint32_t pages_of(const PageParams& p, long long base) {
    const int lane = threadIdx.x & 31;
    const long long first = base + (long long)(threadIdx.x & ~31) * kPer + lane;
    int v[kPer];
#pragma unroll
    for (int j = 0; j < kPer; ++j) v[j] = first + 32 * j < p.P ? __ldcg(p.refs + first + 32 * j) : kFree ? 1 : 0;
    uint32_t mine = 0;
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
        const uint32_t all = __ballot_sync(0xffffffffu, (v[j] == 0) == kFree);
        if (lane >> 1 == j) mine = all;
    }
    return lane & 1 ? mine >> 16 : mine & 0xffffu;
}

// A warp copies piece `piece` of page `src` to page `dst`.
__device__ __forceinline__ void copy_piece(const PagePools& pools, long long src, long long dst, uint32_t piece) {
    int i = 0;
    while (i + 1 < pools.n && pools.first[i + 1] <= piece) ++i;
    const uint32_t vecs = pools.vecs[i], j = (piece - pools.first[i]) * kPiece + (threadIdx.x & 31);
    const uint4* from = pools.data[i] + src * vecs;
    uint4* to = pools.data[i] + dst * vecs;
    uint4 v[kPiece / 32];
#pragma unroll
    for (int k = 0; k < kPiece / 32; ++k)
        if (j + 32 * k < vecs) v[k] = __ldcg(from + j + 32 * k);
#pragma unroll
    for (int k = 0; k < kPiece / 32; ++k)
        if (j + 32 * k < vecs) to[j + 32 * k] = v[k];
}

// ------------------------------------------------------------------- fork
// What request i of a fork asks for.
struct ForkRequest {
    int L, full, own;    // tokens, shared full pages, pages of the new row's own
    int src, dst;
    bool valid;          // src is a row or -1, and dst a row
};
__device__ __forceinline__ ForkRequest fork_request(const PageParams& p, const int32_t* src, const int32_t* dst, int i,
                                                    int room) {
    ForkRequest f;
    f.src = __ldcg(src + i);
    f.dst = __ldcg(dst + i);
    f.valid = f.src >= -1 && f.src < p.R && f.dst >= 0 && f.dst < p.R;
    f.L = f.valid && f.src >= 0 ? clamped_len(p, __ldcg(p.lens + f.src)) : 0;
    f.full = f.L / p.ps;
    const long long end = min((long long)f.L + room, (long long)p.max_pages * p.ps);
    f.own = f.valid ? (int)((end + p.ps - 1) / p.ps) - f.full : 0;
    return f;
}

constexpr int kFindThreads = 1024;

// One CTA: first[i], how many free pages the requests before i ask for, and the
// lowest free pages, as many as all of them ask for (found: how many are listed).
// What is asked for is summed in 64 bits: a request may want 2^30 pages, whatever
// the pool holds.
__global__ void __launch_bounds__(kFindThreads) fork_find_kernel(const PageParams p, const int32_t* src,
                                                                 const int32_t* dst, int n, int room,
                                                                 long long* first, int32_t* free_ids, int* found) {
    __shared__ int s_warp[kFindThreads / 32];
    __shared__ long long s_asked[kFindThreads / 32];
    wait_prior_grid();
    allow_dependent_launch();
    long long want = 0;
    for (long long base = 0; base < n; base += kFindThreads) {
        const long long i = base + threadIdx.x;
        const long long own = i < n ? fork_request(p, src, dst, (int)i, room).own : 0;
        long long total;
        const long long before = block_scan<kFindThreads>(own, s_asked, total);
        if (i < n) first[i] = want + before;
        want += total;
    }
    int have = 0;
    for (long long base = 0; base < p.P && have < want; base += kFindThreads * kPer) {
        const long long id = base + threadIdx.x * kPer;
        uint32_t is_free = pages_of<true>(p, base);
        int total;
        int at = have + block_scan<kFindThreads>(__popc(is_free), s_warp, total);
        for (; is_free; is_free &= is_free - 1, ++at)
            if (at < want) free_ids[at] = (int)(id + __ffs(is_free) - 1);
        have += total;
    }
    if (threadIdx.x == 0) *found = (int)min((long long)have, want);
}

constexpr int kForkThreads = 256;

// CTA (request i, part y): part 0 writes the row, and which page it copies to which
// (-1: none); all parts copy the part-filled page.
__global__ void __launch_bounds__(kForkThreads) fork_row_kernel(const PageParams p, const __grid_constant__ PagePools pools,
                                                                const int32_t* src, const int32_t* dst, int room,
                                                                const long long* first, const int32_t* free_ids,
                                                                const int* found, int32_t* copy_from, int32_t* copy_to,
                                                                int32_t* out_forked) {
    const int i = blockIdx.x;
    wait_prior_grid();
    allow_dependent_launch();
    const ForkRequest f = fork_request(p, src, dst, i, room);
    const long long at = __ldcg(first + i);
    const bool ok = f.valid && at + f.own <= __ldcg(found);
    const int32_t* from = p.table + (size_t)max(f.src, 0) * p.max_pages;
    if (blockIdx.y == 0) {
        if (threadIdx.x == 0) out_forked[i] = ok;
        if (f.dst >= 0 && f.dst < p.R) {
            int32_t* to = p.table + (size_t)f.dst * p.max_pages;
            if (threadIdx.x == 0) p.lens[f.dst] = ok ? f.L : 0;
            for (int j = threadIdx.x; j < p.max_pages; j += kForkThreads) {
                int id = -1;
                if (ok && j < f.full) {
                    id = __ldcg(from + j);
                    if (id >= 0 && id < p.P) atomicAdd(p.refs + id, 1);
                } else if (ok && j < f.full + f.own) {
                    id = __ldcg(free_ids + at + (j - f.full));
                    p.refs[id] = 1;
                }
                to[j] = id;
            }
        }
    }
    int old = -1, to = -1;
    if (ok && f.L % p.ps != 0) {
        old = __ldcg(from + f.full);
        if (old >= 0 && old < p.P) {
            to = __ldcg(free_ids + at);
            constexpr int kWarps = kForkThreads / 32;
            for (uint32_t k = blockIdx.y * kWarps + threadIdx.x / 32; k < pools.pieces; k += gridDim.y * kWarps)
                copy_piece(pools, old, to, k);
        }
    }
    if (blockIdx.y == 0 && threadIdx.x == 0) {
        copy_from[i] = old;
        copy_to[i] = to;
    }
}

// ---------------------------------------------------------------- release
constexpr int kReleaseThreads = 256;

__global__ void __launch_bounds__(kReleaseThreads) release_kernel(const PageParams p, const int32_t* rows,
                                                                  const int32_t* keep_lens) {
    wait_prior_grid();
    allow_dependent_launch();
    const int r = __ldcg(rows + blockIdx.x);
    if (r < 0 || r >= p.R) return;
    const int keep = clamped_len(p, __ldcg(keep_lens + blockIdx.x));
    int32_t* row = p.table + (size_t)r * p.max_pages;
    if (threadIdx.x == 0) p.lens[r] = min(__ldcg(p.lens + r), keep);
    for (int j = (keep + p.ps - 1) / p.ps + threadIdx.x; j < p.max_pages; j += kReleaseThreads) {
        const int id = __ldcg(row + j);
        if (id >= 0 && id < p.P) atomicSub(p.refs + id, 1);
        row[j] = -1;
    }
}

// ---------------------------------------------------------------- compact
constexpr int kCountThreads = 256;
constexpr int kCountTile = kCountThreads * kPer;   // pages a CTA counts

struct CompactParams {
    int* tile_live;      // [tiles] pages in use in each tile of counts; NULL: not counted before
    int32_t* src;        // [P] the moving pages, ascending (as many as move)
    int32_t* dst;        // [P] where they go
    int32_t* rank;       // [P] of an id >= N: its place in src, -1 if it does not move
    int* n_moved;
    int tiles;
};

__global__ void __launch_bounds__(kCountThreads) compact_count_kernel(const PageParams p, const CompactParams c) {
    __shared__ int s_warp[kCountThreads / 32];
    wait_prior_grid();
    allow_dependent_launch();
    int total;
    block_scan<kCountThreads>(__popc(pages_of<false>(p, (long long)blockIdx.x * kCountTile)), s_warp,
                              total);
    if (threadIdx.x == 0) c.tile_live[blockIdx.x] = total;
}

// The place of every page that moves and of every free page that takes one:
// a page in use with id >= N is the (pages in use before it, less those below
// N)-th of the first, a free page below N the (id less pages in use before it)-th
// of the second.
__global__ void __launch_bounds__(kCountThreads) compact_rank_kernel(const PageParams p, const CompactParams c,
                                                                     int32_t* out_live) {
    __shared__ int s_warp[kCountThreads / 32];
    wait_prior_grid();
    allow_dependent_launch();
    auto sum = [&](int v) {
        int total;
        block_scan<kCountThreads>(v, s_warp, total);
        return total;
    };
    const long long mine = (long long)blockIdx.x * kCountTile, id0 = mine + threadIdx.x * kPer;
    const uint32_t own = pages_of<false>(p, mine);
    auto live_of = [&](long long base) { return base == mine ? own : pages_of<false>(p, base); };
    // f(the pages in use of a stretch, its first id): stretches of a tile, or, where
    // they are not counted before, of a thread's counts
    auto each = [&](auto f) {
        if (c.tile_live) {
            for (int t = threadIdx.x; t < c.tiles; t += kCountThreads) f(__ldcg(c.tile_live + t), (long long)t * kCountTile);
        } else {
            for (long long base = 0; base < p.P; base += kCountTile) f(__popc(live_of(base)), base + threadIdx.x * kPer);
        }
    };
    int before = 0, all = 0;
    each([&](int live, long long id) {
        all += live;
        if (id < mine) before += live;
    });
    const int N = sum(all);
    before = sum(before);
    // pages in use below N: the stretches that end there, and the one that N lies in
    const int stretch = c.tile_live ? kCountTile : kPer;
    int below = 0;
    each([&](int live, long long id) {
        if (id + stretch <= N) below += live;
    });
    {
        const long long base = (long long)N / kCountTile * kCountTile, id = base + threadIdx.x * kPer;
        const uint32_t live = live_of(base);
#pragma unroll
        for (int j = 0; j < kPer; ++j)
            if (id + j >= (long long)N / stretch * stretch && id + j < N && (live >> j & 1)) ++below;
    }
    below = sum(below);
    int total;
    int at = before + block_scan<kCountThreads>(__popc(own), s_warp, total);
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
        const int id = (int)(id0 + j);
        if (id0 + j >= p.P) break;
        const bool on = own >> j & 1;
        if (id < N && !on) c.dst[id - at] = id;
        if (id >= N) {
            c.rank[id] = on ? at - below : -1;
            if (on) c.src[at - below] = id;
        }
        at += on;
    }
    if (blockIdx.x == 0 && threadIdx.x == 0) {
        *out_live = N;
        *c.n_moved = N - below;
    }
}

constexpr int kMoveThreads = 256;

// The first `copy_ctas` CTAs copy pages, a warp a piece at a time (a CTA a page:
// 239 pages of 64 KB took 28 us, 26,637 of 18 KB 250), the others rename table
// entries.
__global__ void __launch_bounds__(kMoveThreads) compact_move_kernel(const PageParams p,
                                                                    const __grid_constant__ PagePools pools,
                                                                    const CompactParams c, const int32_t* live,
                                                                    int copy_ctas) {
    wait_prior_grid();
    allow_dependent_launch();
    if ((int)blockIdx.x < copy_ctas) {
        const int moved = __ldcg(c.n_moved);
        const uint32_t pieces = max(pools.pieces, 1u);   // (no pool: the counts alone)
        const long long items = (long long)moved * pieces, step = (long long)copy_ctas * (kMoveThreads / 32);
        for (long long it = (long long)blockIdx.x * (kMoveThreads / 32) + threadIdx.x / 32; it < items; it += step) {
            const long long r = div_pos(it, pieces);
            const uint32_t k = (uint32_t)(it - r * pieces);
            const int from = __ldcg(c.src + r), to = __ldcg(c.dst + r);
            if (k < pools.pieces) copy_piece(pools, from, to, k);
            if (k == 0 && (threadIdx.x & 31) == 0) {
                p.refs[to] = __ldcg(p.refs + from);
                p.refs[from] = 0;
            }
        }
        return;
    }
    const int N = __ldcg(live);
    const long long entries = (long long)p.R * p.max_pages;
    for (long long e = (long long)(blockIdx.x - copy_ctas) * kMoveThreads + threadIdx.x; e < entries;
         e += (long long)(gridDim.x - copy_ctas) * kMoveThreads) {
        const int id = __ldcg(p.table + e);
        if (id < N || id >= p.P) continue;
        const int r = __ldcg(c.rank + id);
        if (r >= 0) p.table[e] = __ldcg(c.dst + r);
    }
}

// The copies of a fork or a compaction in further pools: page from[r] to page to[r], r
// below n and *count (NULL: n).  What is no page is left out, whatever the lists hold.
__global__ void __launch_bounds__(kMoveThreads) copy_more_kernel(const __grid_constant__ PagePools pools,
                                                                 const int32_t* from, const int32_t* to,
                                                                 const int* count, int n, int P) {
    wait_prior_grid();
    allow_dependent_launch();
    const int copies = count ? min(n, __ldcg(count)) : n;
    const long long items = (long long)copies * pools.pieces, step = (long long)gridDim.x * (kMoveThreads / 32);
    for (long long it = (long long)blockIdx.x * (kMoveThreads / 32) + threadIdx.x / 32; it < items; it += step) {
        const long long r = div_pos(it, pools.pieces);
        const int a = __ldcg(from + r), b = __ldcg(to + r);
        if (a >= 0 && a < P && b >= 0 && b < P && a != b) copy_piece(pools, a, b, (uint32_t)(it - r * pools.pieces));
    }
}

size_t align256(size_t n) { return (n + 255) & ~size_t(255); }

PageParams page_params(const cs_page_dims& d, int32_t* table, int32_t* lens, int32_t* refs) {
    PageParams p{};
    p.table = table;
    p.lens = lens;
    p.refs = refs;
    p.R = d.rows;
    p.max_pages = d.max_pages_per_seq;
    p.ps = d.page_size;
    p.P = d.num_pages;
    return p;
}

PagePools page_pools(const cs_page_pool* pools, int n) {
    PagePools q{};
    for (int i = 0; i < n; ++i) {
        q.data[i] = static_cast<uint4*>(pools[i].data);
        q.vecs[i] = (uint32_t)(pools[i].page_bytes / 16);
        q.first[i] = q.pieces;
        q.pieces += (q.vecs[i] + kPiece - 1) / kPiece;
    }
    q.n = n;
    return q;
}

int tiles_of_counts(int P) { return (int)(((long long)P + kCountTile - 1) / kCountTile); }

}  // namespace

// found (256 B), first [n], the copied pages and where they go [n], the free pages (at most all)
size_t fork_workspace_bytes(const cs_page_dims& d, int n) {
    return 256 + align256(sizeof(long long) * (size_t)n) + 2 * align256(sizeof(int32_t) * (size_t)n) +
           align256(sizeof(int32_t) * (size_t)d.num_pages);
}

namespace {
struct ForkSpace {
    int* found;
    long long* first;
    int32_t *copy_from, *copy_to, *free_ids;
    ForkSpace(void* workspace, int n) {
        uint8_t* ws = static_cast<uint8_t*>(workspace);
        const size_t ids = align256(sizeof(int32_t) * (size_t)n);
        found = reinterpret_cast<int*>(ws);
        first = reinterpret_cast<long long*>(ws + 256);
        ws += 256 + align256(sizeof(long long) * (size_t)n);
        copy_from = reinterpret_cast<int32_t*>(ws);
        copy_to = reinterpret_cast<int32_t*>(ws + ids);
        free_ids = reinterpret_cast<int32_t*>(ws + 2 * ids);
    }
};

cs_status launch_copy_more(const cs_page_dims& d, const cs_page_pool* pools, int n_pools, const int32_t* from,
                           const int32_t* to, const int* count, int n, cudaStream_t stream) {
    const cudaError_t e = launch_dependent(copy_more_kernel, dim3(7 * current_sm_count()), dim3(kMoveThreads), 0, stream,
                                           page_pools(pools, n_pools), from, to, count, n, (int)d.num_pages);
    return e == cudaSuccess ? CS_OK : cuda_fail(e, "copy_more_kernel launch");
}
}  // namespace

cs_status launch_kv_fork(const cs_page_dims& d, const cs_page_pool* pools, int n_pools, int32_t* page_table,
                         int32_t* ctx_lens, int32_t* ref_counts, const int32_t* src, const int32_t* dst, int n,
                         int room, int32_t* out_forked, void* workspace, cudaStream_t stream) {
    const ForkSpace ws(workspace, n);
    const PageParams p = page_params(d, page_table, ctx_lens, ref_counts);
    cudaError_t e = launch_dependent(fork_find_kernel, dim3(1), dim3(kFindThreads), 0, stream, p, src, dst, n, room,
                                     ws.first, ws.free_ids, ws.found);
    if (e != cudaSuccess) return cuda_fail(e, "fork_find_kernel launch");
    const PagePools q = page_pools(pools, n_pools);
    // a warp some four pieces of the page that is copied
    const unsigned parts = q.pieces / 32 < 1 ? 1 : q.pieces / 32 > 32 ? 32 : q.pieces / 32;
    e = launch_dependent(fork_row_kernel, dim3(n, parts), dim3(kForkThreads), 0, stream, p, q, src,
                         dst, room, (const long long*)ws.first, (const int32_t*)ws.free_ids, (const int*)ws.found,
                         ws.copy_from, ws.copy_to, out_forked);
    return e == cudaSuccess ? CS_OK : cuda_fail(e, "fork_row_kernel launch");
}

cs_status launch_kv_fork_more(const cs_page_dims& d, const cs_page_pool* pools, int n_pools, int n, void* workspace,
                              cudaStream_t stream) {
    const ForkSpace ws(workspace, n);
    return launch_copy_more(d, pools, n_pools, ws.copy_from, ws.copy_to, nullptr, n, stream);
}

cs_status launch_kv_release(const cs_page_dims& d, int32_t* page_table, int32_t* ctx_lens, int32_t* ref_counts,
                            const int32_t* rows, const int32_t* keep_lens, int n, cudaStream_t stream) {
    const cudaError_t e = launch_dependent(release_kernel, dim3(n), dim3(kReleaseThreads), 0, stream,
                                           page_params(d, page_table, ctx_lens, ref_counts), rows, keep_lens);
    return e == cudaSuccess ? CS_OK : cuda_fail(e, "release_kernel launch");
}

// n_moved (256 B), tile counts, src, dst, rank
size_t compact_workspace_bytes(const cs_page_dims& d) {
    return 256 + align256(sizeof(int) * (size_t)tiles_of_counts(d.num_pages)) +
           3 * align256(sizeof(int32_t) * (size_t)d.num_pages);
}

namespace {
CompactParams compact_params(const cs_page_dims& d, void* workspace) {
    uint8_t* ws = static_cast<uint8_t*>(workspace);
    const size_t ids = align256(sizeof(int32_t) * (size_t)d.num_pages);
    CompactParams c{};
    c.tiles = tiles_of_counts(d.num_pages);
    c.n_moved = reinterpret_cast<int*>(ws);
    c.tile_live = reinterpret_cast<int*>(ws + 256);
    ws += 256 + align256(sizeof(int) * (size_t)c.tiles);
    c.src = reinterpret_cast<int32_t*>(ws);
    c.dst = reinterpret_cast<int32_t*>(ws + ids);
    c.rank = reinterpret_cast<int32_t*>(ws + 2 * ids);
    return c;
}
}  // namespace

cs_status launch_kv_compact(const cs_page_dims& d, const cs_page_pool* pools, int n_pools, int32_t* page_table,
                            int32_t* ref_counts, int32_t* out_live, void* workspace, cudaStream_t stream) {
    CompactParams c = compact_params(d, workspace);
    const PageParams p = page_params(d, page_table, nullptr, ref_counts);
    cudaError_t e = cudaSuccess;
    // up to four tiles the ranking counts them itself: a launch less
    if (c.tiles <= 4) {
        c.tile_live = nullptr;
    } else {
        e = launch_dependent(compact_count_kernel, dim3(c.tiles), dim3(kCountThreads), 0, stream, p, c);
        if (e != cudaSuccess) return cuda_fail(e, "compact_count_kernel launch");
    }
    e = launch_dependent(compact_rank_kernel, dim3(c.tiles), dim3(kCountThreads), 0, stream, p, c, out_live);
    if (e != cudaSuccess) return cuda_fail(e, "compact_rank_kernel launch");
    const int sms = current_sm_count();
    e = launch_dependent(compact_move_kernel, dim3(8 * sms), dim3(kMoveThreads), 0, stream, p, page_pools(pools, n_pools),
                         c, (const int32_t*)out_live, 7 * sms);
    return e == cudaSuccess ? CS_OK : cuda_fail(e, "compact_move_kernel launch");
}

cs_status launch_kv_compact_more(const cs_page_dims& d, const cs_page_pool* pools, int n_pools, void* workspace,
                                 cudaStream_t stream) {
    const CompactParams c = compact_params(d, workspace);
    return launch_copy_more(d, pools, n_pools, c.src, c.dst, c.n_moved, d.num_pages, stream);
}

}  // namespace cs
