// packed_attention_tc.cuh -- the tcgen05 form of packed attention, for 33 to 80
// query rows of a span (included by packed_attention.cu inside its anonymous
// namespace: the same split of the keys, pieces and merge).
//
// Transposed products, so that the padding is to 16 query rows (N) and the keys
// and dims fill M = 128:
//   S^T [128 keys x N] = K Q^T    K as fp16 in tensor memory (a thread decodes
//       the row of its key, its lane), Q a K-major shared-memory operand;
//   O^T [128 dims x N] += V^T P^T  V as fp16 and P in shared memory, both
//       MN-major: a thread writes the row of its key as it is.
//
// Two CTAs an SM of eight warps, each with one buffer of
// everything: while one waits for a product, a fence or a vote, the other has
// the SM.  (A ninth warp for the MMAs counts as four when the SM's registers
// are shared out: one CTA fits then.)  Warps 0-3 decode the K rows of a tile, warps 4-7 its V rows; the
// codes of the next tile come by cp.async meanwhile, every thread's own row.
// Then all eight do the softmax, a thread one key and each four warps a share
// of the columns (query rows).  Warp 0 issues the product for S, warp 4 that for
// O: each would wait for it next.
//
// As in the other form P = 2^(s - m + 12), and the tile is taken the short way
// unless some weight would leave [2^-14, 2^15] (a vote of the workers).  Then
// (mend) the columns' maxima are found, O is rescaled where one grows by more than
// 2^3, and weights below 2^-14 (faint) are taken 28 powers of two at a time by
// products of their own, which the workers add to O.  Mending is rolled up, for
// the instruction cache's sake.
//
// Every mbarrier wait is bounded; after one that gives up nothing waits or is
// issued any more, every warp still meets every block barrier, and the status
// word says so.

constexpr int kTcThreads = 256;
constexpr int kTcTile = 128;                       // keys of a tile: the MMAs' M (S) and K (O)
constexpr int kTcVBytes = kTcTile * 256;           // V of a tile in fp16
constexpr int kTcRawBytes = 2 * kTcTile * kPackCodeBytes;   // codes of K and V of a tile
constexpr int kTcMaxRows = 80;                     // query rows of a span at most

template <int kN>
struct TcForm {
    static constexpr int kMinBlocks = 2;
    static constexpr int kH = (kN + 15) / 16 * 8, kH1 = kN - kH;         // columns of warps 0-3, of warps 4-7: multiples of 8
    static constexpr int kAtoms = kN > 64 ? 2 : 1;                       // 64-column atoms of P
    static constexpr int kPGroup = kAtoms * 1024;                        // bytes of P for 8 keys
    static constexpr int kQHalf = kN * 128;                              // bytes of a dim half of Q
    static constexpr int kColS = 64, kColO = kColS + kN;                 // tensor memory: K [0, 64), S, O
    static constexpr int kCols = kColO + kN <= 128 ? 128 : 256;
    static_assert(kColO + kN <= kCols && kCols * kMinBlocks <= 512, "tensor memory");
    // V | P | Q | raw codes | columns | lengths
    static constexpr int kOffP = kTcVBytes, kOffQ = kOffP + kTcTile / 8 * kPGroup, kOffRaw = kOffQ + 2 * kQHalf;
    static constexpr int kOffCol = kOffRaw + kTcRawBytes, kOffLen = kOffCol + kN * 4 * (5 + 8);
    static constexpr int kSmem = kOffLen + kMaxBatchPerLaunch * 4 + 1024;
    static_assert((kSmem + 2048) * kMinBlocks <= 233472, "shared memory");
};

__device__ __forceinline__ void tc_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tc_wait_ld() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void fence_async_smem() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

// 8 columns of the warp's 32 lanes (complete after tc_wait_ld)
__device__ __forceinline__ void tc_ld8(uint32_t addr, float* v) {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
                 : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]), "=f"(v[4]), "=f"(v[5]), "=f"(v[6]), "=f"(v[7])
                 : "r"(addr));
}
__device__ __forceinline__ void tc_st8(uint32_t addr, const uint32_t* r) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"r"(addr), "r"(r[0]), "r"(r[1]),
                 "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7])
                 : "memory");
}
__device__ __forceinline__ void tc_st16(uint32_t addr, const uint32_t* r) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};" ::"r"(
            addr),
        "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]),
        "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
        : "memory");
}

__device__ __forceinline__ void tc_mma_ss(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t acc) {
    asm volatile(
        "{\n\t.reg .pred q;\n\tsetp.ne.b32 q, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, q;\n\t}\n" ::"r"(d),
        "l"(a), "l"(b), "r"(idesc), "r"(acc)
        : "memory");
}

// 128-byte swizzle, 8-row (K-major) or 8-key (MN-major) groups `group` bytes
// apart, 64-element atoms of an MN-major operand `atom` bytes apart
__device__ __forceinline__ uint64_t tc_desc(uint32_t addr, uint32_t group, uint32_t atom) {
    return (uint64_t)((addr >> 4) & 0x3FFF) | ((uint64_t)(atom >> 4) << 16) | ((uint64_t)(group >> 4) << 32) |
           (1ull << 46) | (2ull << 61);
}
// kind::f16, both operands fp16, fp32 sums, M = 128, N = n
__host__ __device__ constexpr uint32_t tc_idesc(int n, bool a_mn, bool b_mn) {
    return (1u << 4) | (a_mn ? 1u << 15 : 0u) | (b_mn ? 1u << 16 : 0u) | ((uint32_t)(n >> 3) << 17) | (8u << 24);
}

// Whether any of the workers' threads says so; a barrier of theirs.
__device__ __forceinline__ bool workers_any(bool x) {
    uint32_t r;
    asm volatile(
        "{\n\t.reg .pred p, q;\n\tsetp.ne.u32 p, %1, 0;\n\tbarrier.cta.red.or.pred q, 1, 256, p;\n\t"
        "selp.u32 %0, 1, 0, q;\n\t}\n"
        : "=r"(r)
        : "r"((uint32_t)x)
        : "memory");
    return r != 0;
}
__device__ __forceinline__ void workers_sync() { asm volatile("barrier.cta.sync 1, 256;" ::: "memory"); }

// A float's bits as an integer of the same order, and back.
__device__ __forceinline__ int ordered(float x) {
    const int b = __float_as_int(x);
    return b < 0 ? b ^ 0x7fffffff : b;
}
__device__ __forceinline__ float unordered(int b) { return __int_as_float(b < 0 ? b ^ 0x7fffffff : b); }

// Waits for the phase of the given parity, asleep for up to 20 us.
__device__ __forceinline__ bool tc_asleep(uint64_t* bar, uint32_t parity) {
    uint32_t done;
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2, 20000;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}\n"
        : "=r"(done)
        : "r"(smem_u32(bar)), "r"(parity)
        : "memory");
    return done != 0;
}
// Bounded (about one second); returns at once when another wait has given up.
// (Out of line: the loop's code is long.)
__device__ __noinline__ void tc_wait_long(uint64_t* bar, uint32_t parity, volatile int* dead, int* status) {
    const uint64_t t0 = global_timer_ns();
    while (!*dead) {
        if (tc_asleep(bar, parity)) return;
        if (global_timer_ns() - t0 > 1000000000ull) {
            *dead = 1;
            atomicOr(status, CS_DEVICE_WAIT_TIMEOUT);
        }
    }
}
__device__ __forceinline__ void tc_wait(uint64_t* bar, uint32_t parity, volatile int* dead, int* status) {
    if (!tc_asleep(bar, parity)) tc_wait_long(bar, parity, dead, status);
}
// Whether no wait has given up, the same answer in the whole warp.
__device__ __forceinline__ bool alive(volatile int* dead) { return !__any_sync(0xffffffffu, *dead); }

struct TcBars {
    uint64_t k_full;       // K of a tile decoded (4 warps)
    uint64_t s_full;       // S of a tile done; its K is read
    uint64_t p_full;       // P and V of a tile written, its S read (8 warps)
    uint64_t o_done;       // O of a tile done; its P and V are read
    uint64_t f_done;       // a product of faint weights done
};

// V^T P^T, n columns of P from an atom's first on, into the columns from d on
// (one thread issues): 8 steps of 16 keys.
template <int kN>
__device__ __forceinline__ void tc_mma_values(uint32_t d, uint8_t* smem, int atom, int n, bool add) {
    using F = TcForm<kN>;
    const uint32_t id = tc_idesc(n, true, true);
    const uint64_t v = tc_desc(smem_u32(smem), 2048, 1024);
    const uint64_t x = tc_desc(smem_u32(smem + F::kOffP + atom * 1024), F::kPGroup, 1024);
#pragma unroll
    for (int kk = 0; kk < kTcTile / 16; ++kk)
        tc_mma_ss(d, v + (uint64_t)(kk * (4096 >> 4)), x + (uint64_t)(kk * 2 * F::kPGroup >> 4), id, add || kk > 0 ? 1u : 0u);
}

template <int kN>
__device__ __forceinline__ void tc_worker(const PackedAttnParams& p, uint8_t* smem, TcBars& bars, uint32_t tmem,
                                          volatile int* dead, const int* s_info, const int* s_len, const Cursor start,
                                          const int n_tiles, const int* s_draft) {
    using F = TcForm<kN>;
    constexpr int kH = F::kH;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, quad = warp & 3;
    const bool v_side = warp >= 4;
    // this side's columns: kH of them, or fewer (one body of code for both)
    const int kC0 = v_side ? kH : 0, n_cols = v_side ? F::kH1 : kH;
    auto mine = [&](int i) { return kH == F::kH1 || i < n_cols; };
    const int key = 32 * quad + lane;                    // of a tile; also the lane of tensor memory
    const uint32_t lanes = (uint32_t)(32 * quad) << 16;
    const int nb = p.n_batch, cta = blockIdx.x;
    float* s_sc = reinterpret_cast<float*>(smem + F::kOffCol);   // [N] scale of a column's scores
    float* s_up = s_sc + kN;                             // [N] 12 - m
    float* s_alpha = s_up + kN;                          // [N] what a column's sums are rescaled by
    float* s_m = s_alpha + kN;                           // [N] running maxima
    float* s_inv = s_m + kN;                             // [N] 1 / l at the end
    int* s_red = reinterpret_cast<int*>(s_inv + kN);     // [4][N] the quads' maxima, or sums
    float* s_faint = reinterpret_cast<float*>(s_red + 4 * kN);   // [4][N] the quads' sums of faint weights

    uint8_t* s_q = smem + F::kOffQ;

    // ---- the next tile's row: codes into shared memory (parts exchanged by the
    // key's bits, so that the threads' 16-byte loads meet every bank once), scales
    const uint8_t* codes = v_side ? p.v_codes : p.k_codes;
    const uint8_t* scales = v_side ? p.v_scales : p.k_scales;
    uint8_t* const raw = smem + F::kOffRaw + (v_side ? kTcRawBytes / 2 : 0) + key * kPackCodeBytes;
    const int raw_x = (key >> 1) & 3;
    Cursor cl = start;           // the tile whose page is looked up next
    int left = n_tiles;
    int page = -1, slot = 0;     // of the tile whose row is loaded next
    uint2 sc8 = make_uint2(0, 0);
    auto look_up = [&]() {
        page = -1;
        if (left <= 0) return;
        --left;
        const int pos = cl.t * kTcTile + key;
        slot = (p.n_rb == 1 ? cl.h : cl.h / p.n_rb) * p.ps + (pos & (p.ps - 1));
        if (pos < s_len[cl.b])
            page = __ldcg(p.page_table + (size_t)(p.b_base + cl.b) * p.max_pages + (pos >> p.ps_log2));
        advance(cl, s_len, nb, p.n_spans, kTcTile);
    };
    auto load_row = [&]() {      // zeros for a key past the context or on no page
        const bool in = page >= 0 && page < p.P;
        const size_t row = in ? (size_t)page * p.Hkv * p.ps + slot : 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) cp_async16(smem_u32(raw + ((i ^ raw_x) << 4)), codes + row * kPackCodeBytes + 16 * i, in);
        cp_async_commit();
        sc8 = in ? __ldcg(reinterpret_cast<const uint2*>(scales + row * kPackGroups)) : make_uint2(0, 0);
        look_up();
    };
    // the row as fp16, into tensor memory (K) or shared memory (V)
    uint8_t* const v_row = smem + (key >> 3) * 2048 + (key & 7) * 128;
    auto decode = [&]() {
        cp_async_wait<0>();
#pragma unroll
        for (int i = 0; i < 4; ++i) {   // 32 dims: 16 pairs
            const uint4 w4 = *reinterpret_cast<const uint4*>(raw + ((i ^ raw_x) << 4));
            const uint32_t w[4] = {w4.x, w4.y, w4.z, w4.w};
            const uint32_t f = scales_f16x2((i & 2 ? sc8.y : sc8.x) >> (i & 1 ? 16 : 0));
            uint32_t x[16];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const uint32_t s = __byte_perm(f, 0, j < 2 ? 0x1010 : 0x3232);
                x[4 * j] = mul_f16x2(codes_f16x2<0>(w[j]), s);
                x[4 * j + 1] = mul_f16x2(codes_f16x2<1>(w[j]), s);
                x[4 * j + 2] = mul_f16x2(codes_f16x2<2>(w[j]), s);
                x[4 * j + 3] = mul_f16x2(codes_f16x2<3>(w[j]), s);
            }
            if (!v_side) {
                tc_st16(tmem + lanes + 16 * i, x);
            } else {
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    *reinterpret_cast<uint4*>(v_row + (i >> 1) * 1024 + ((((i & 1) * 4 + j) ^ (key & 7)) << 4)) =
                        make_uint4(x[4 * j], x[4 * j + 1], x[4 * j + 2], x[4 * j + 3]);
            }
        }
    };
    // eight of a key's columns of P, from `col` on
    uint8_t* const p_row = smem + F::kOffP + (key >> 3) * F::kPGroup + (key & 7) * 128;
    auto store_p = [&](int col, uint32_t x0, uint32_t x1, uint32_t x2, uint32_t x3) {
        *reinterpret_cast<uint4*>(p_row + (col >> 6) * 1024 + ((((col & 63) >> 3) ^ (key & 7)) << 4)) =
            make_uint4(x0, x1, x2, x3);
    };

    look_up();
    load_row();
    Cursor cur = start;
    float l[kH];
    bool first_piece = true;
    uint32_t f_phase = 0;
    int piece_t0 = cur.t;
#pragma unroll 1
    for (int j = 0; j < n_tiles; ++j) {
        const int L = s_len[cur.b], bg = p.b_base + cur.b;
        // the KV head of the span, and its row block's first row
        const int head = p.n_rb == 1 ? cur.h : cur.h / p.n_rb, row0 = (cur.h - head * p.n_rb) * p.n_rows;
        const int n_live = min(p.n_rows, p.n_all - row0);
        const uint32_t ph = (uint32_t)j & 1;
        const bool first = j == 0 || cur.t == 0, last = j + 1 == n_tiles || cur.t + 1 == cur.T;
        if (first) {
            // ---- a new piece: its query rows as fp16 below 2^15 (as in the other form)
            piece_t0 = cur.t;
#pragma unroll
            for (int i = 0; i < kH; ++i) l[i] = 0.f;
            constexpr int kMine = kN / 8;   // rows of a warp, requested together
            uint2 x[kMine];
            const float scale = p.scale_log2 * (p.k_head ? __ldcg(p.k_head + head) : 1.f);
#pragma unroll
            for (int k = 0; k < kMine; ++k) {
                const int row = warp + 8 * k;
                x[k] = make_uint2(0, 0);
                if (row < n_live) {
                    const int i = s_draft[row0 + row];
                    const uint32_t* src = reinterpret_cast<const uint32_t*>(
                        p.q + (((size_t)bg * p.R + i) * p.Hq + (size_t)head * p.G + (row0 + row - i * p.G)) * kPackDim + 4 * lane);
                    x[k].x = __ldcg(src);
                    x[k].y = __ldcg(src + 1);
                }
            }
#pragma unroll
            for (int k = 0; k < kMine; ++k) {
                const int row = warp + 8 * k;
                float back;
                const uint2 y = query_f16(x[k], back);
                *reinterpret_cast<uint2*>(s_q + (lane >> 4) * F::kQHalf + row * 128 +
                                          ((((lane & 15) >> 1) ^ (row & 7)) << 4) + (lane & 1) * 8) = y;
                if (lane == 0) {
                    // (not 0, under which a hidden score would be NaN)
                    s_sc[row] = row < n_live ? fmaxf(scale * back, 0x1p-126f) : 0x1p-126f;
                    s_up[row] = row < n_live ? -kNegInf : 0.f;
                    s_m[row] = row < n_live ? kNegInf : kPUp;
                    for (int k4 = 0; k4 < 4; ++k4) s_faint[k4 * kN + row] = 0.f;
                }
            }
            fence_async_smem();
            workers_sync();
        }
        // ---- this tile's row (V once the product of the tile before has read its buffer),
        // and the request of the next one's
        if (v_side && j > 0) tc_wait(&bars.o_done, ph ^ 1, dead, p.status);
        decode();
        load_row();
        if (!v_side) {
            tc_wait_st();
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(&bars.k_full);
            if (warp == 0) {
                // (each wait names the phase that follows the last one seen of its barrier)
                tc_wait(&bars.k_full, ph, dead, p.status);
                tc_fence_after();
                __syncwarp();
                if (alive(dead) && elect_one()) {
                    const uint64_t dq = tc_desc(smem_u32(s_q), 1024, 0);
#pragma unroll
                    for (int ks = 0; ks < kPackDim / 16; ++ks)
                        tc_mma_ts(tmem + F::kColS, tmem + ks * 8,
                                  dq + (uint64_t)((ks >> 2) * (F::kQHalf >> 4) + (ks & 3) * 2), tc_idesc(kN, false, false),
                                  ks > 0 ? 1u : 0u);
                    tc_commit(&bars.s_full);
                }
                __syncwarp();
            }
        }
        // ---- softmax: this key's scores
        tc_wait(&bars.s_full, ph, dead, p.status);
        tc_fence_after();
        const uint32_t s_at = tmem + lanes + F::kColS + kC0, o_at = tmem + lanes + F::kColO + kC0;
        const int key0 = cur.t * kTcTile;
        // the columns that do not see this thread's key: all past the context, else those
        // of the drafts before it (columns are drafts in order, G query heads each)
        const bool edge = key0 + kTcTile > L - p.R + 1;
        const int hidden = !edge ? 0 : key0 + key >= L ? kN : (key0 + key - (L - p.R)) * p.G - row0;
        bool starts = first;   // whether the tile's product starts O
        // what a tile needs before it can go the short way
        auto mend = [&]() {
#pragma unroll 1
            for (int i = 0; i < n_cols; i += 8) {
                float z[8];
                tc_ld8(s_at + i, z);
                tc_wait_ld();
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    const int row = kC0 + i + k;
                    const int top = __reduce_max_sync(0xffffffffu, ordered(row < hidden ? kNegInf : z[k] * s_sc[row]));
                    if (lane == 0) s_red[quad * kN + row] = top;
                }
            }
            workers_sync();
            bool grew = false;
            if (key < n_cols) {
                const int row = kC0 + key;
                const float now = unordered(max(max(s_red[row], s_red[kN + row]), max(s_red[2 * kN + row], s_red[3 * kN + row])));
                const float m = s_m[row];
                float a = 1.f;
                if (row < n_live && now - m > kPMax - kPUp) {   // (true for the first key: m is -inf)
                    a = ex2(m - now);
                    s_m[row] = now;
                    s_up[row] = kPUp - now;
                    for (int k = 0; k < 4; ++k) s_faint[k * kN + row] *= a;
                    grew = !first;
                } else if (m == kNegInf) {
                    s_up[row] = 0.f;   // (no key for this row in the piece: those that a row sees come first)
                }
                s_alpha[row] = a;
            }
            const bool rescale = workers_any(grew);
#pragma unroll
            for (int i = 0; i < kH; i += 4) {
                if (!mine(i)) continue;
                const float4 a = *reinterpret_cast<const float4*>(s_alpha + kC0 + i);
                l[i] *= a.x;
                l[i + 1] *= a.y;
                l[i + 2] *= a.z;
                l[i + 3] *= a.w;
            }
            auto is_faint = [&](float x) { return x < kPMin && x > kPGone; };
            bool faint = false;
#pragma unroll 1
            for (int i = 0; i < n_cols; i += 8) {
                float z[8];
                tc_ld8(s_at + i, z);
                tc_wait_ld();
#pragma unroll
                for (int k = 0; k < 8; ++k)
                    faint |= kC0 + i + k >= hidden && is_faint(fmaf(z[k], s_sc[kC0 + i + k], s_up[kC0 + i + k]));
            }
            faint = workers_any(faint);
            if ((rescale || faint) && j > 0) {
                tc_wait(&bars.o_done, ph ^ 1, dead, p.status);
                tc_fence_after();
            }
            if (rescale) {
#pragma unroll 1
                for (int i = 0; i < n_cols; i += 8) {
                    float o[8];
                    tc_ld8(o_at + i, o);
                    tc_wait_ld();
#pragma unroll
                    for (int k = 0; k < 8; ++k) o[k] *= s_alpha[kC0 + i + k];
                    tc_st8(o_at + i, reinterpret_cast<const uint32_t*>(o));
                }
                tc_wait_st();
            }
#pragma unroll 1
            for (float up = 28.f; faint; up += 28.f) {
                bool more = false;
#pragma unroll 1
                for (int i = 0; i < n_cols; i += 8) {   // this turn's weights, which then are done
                    float z[8], f[8];
                    tc_ld8(s_at + i, z);
                    tc_wait_ld();
#pragma unroll
                    for (int k = 0; k < 8; ++k) {
                        const int row = kC0 + i + k;
                        const float x = fmaf(z[k], s_sc[row], s_up[row]);
                        const bool seen = row >= hidden, now = seen && x < kPMin && x + up >= kPMin;
                        f[k] = now ? ex2(x + up) : 0.f;
                        more |= seen && !now && is_faint(x);
                        if (now) z[k] = kNegInf;
                        float sum = now ? ex2(x) : 0.f;
#pragma unroll
                        for (int off = 16; off > 0; off >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, off);
                        if (lane == 0) s_faint[quad * kN + row] += sum;
                    }
                    tc_st8(s_at + i, reinterpret_cast<const uint32_t*>(z));
                    store_p(kC0 + i, pack_f16x2(f[0], f[1]), pack_f16x2(f[2], f[3]), pack_f16x2(f[4], f[5]),
                            pack_f16x2(f[6], f[7]));
                }
                tc_wait_st();
                fence_async_smem();
                const float down = ex2(-up);
#pragma unroll 1
                for (int atom = 0; atom < F::kAtoms; ++atom) {   // 64 columns at a time, into the place of this tile's K
                    tc_fence_before();
                    workers_sync();
                    tc_fence_after();
                    if (warp == 0 && alive(dead) && elect_one()) {
                        tc_mma_values<kN>(tmem, smem, atom, min(64, kN - 64 * atom), false);
                        tc_commit(&bars.f_done);
                    }
                    __syncwarp();
                    tc_wait(&bars.f_done, f_phase, dead, p.status);
                    f_phase ^= 1;
                    tc_fence_after();
#pragma unroll 1
                    for (int i = 0; i < n_cols; i += 8) {
                        if ((kC0 + i) >> 6 != atom) continue;
                        float o[8], f[8];
                        tc_ld8(tmem + lanes + ((kC0 + i) & 63), f);
                        tc_ld8(o_at + i, o);
                        tc_wait_ld();
                        // (a piece's first tile finds no sums yet)
#pragma unroll
                        for (int k = 0; k < 8; ++k) o[k] = starts ? f[k] * down : fmaf(f[k], down, o[k]);
                        tc_st8(o_at + i, reinterpret_cast<const uint32_t*>(o));
                    }
                    tc_wait_st();
                }
                starts = false;
                tc_fence_before();
                faint = workers_any(more);
                tc_fence_after();
            }
        };
        // x = s - m + 12 of this side's columns, eight at a time
        auto scores = [&](int i, float (&x)[8]) {
            tc_ld8(s_at + i, x);
            float c[8], u[8];
#pragma unroll
            for (int k = 0; k < 8; k += 4) {
                *reinterpret_cast<float4*>(c + k) = *reinterpret_cast<const float4*>(s_sc + kC0 + i + k);
                *reinterpret_cast<float4*>(u + k) = *reinterpret_cast<const float4*>(s_up + kC0 + i + k);
            }
            tc_wait_ld();
#pragma unroll
            for (int k = 0; k < 8; k += 2)
                f2_unpack(f2_fma(f2_pack(x[k], x[k + 1]), f2_pack(c[k], c[k + 1]), f2_pack(u[k], u[k + 1])), x[k], x[k + 1]);
        };
        float most = 0.f, least = 0.f;
#pragma unroll
        for (int i = 0; i < kH; i += 8) {
            if (!mine(i)) continue;
            float x[8];
            scores(i, x);
            if (edge)
#pragma unroll
                for (int k = 0; k < 8; ++k) x[k] = kC0 + i + k < hidden ? 0.f : x[k];
#pragma unroll
            for (int k = 0; k < 8; k += 2) {
                most = fmax3(most, x[k], x[k + 1]);
                least = fmin3(least, x[k], x[k + 1]);
            }
        }
        if (workers_any(most > kPMax || least < kPMin)) mend();
        if (!v_side && j > 0) tc_wait(&bars.o_done, ph ^ 1, dead, p.status);   // P is free
#pragma unroll
        for (int i = 0; i < kH; i += 8) {
            if (!mine(i)) continue;
            float x[8];
            scores(i, x);
            if (edge)
#pragma unroll
                for (int k = 0; k < 8; ++k) x[k] = kC0 + i + k < hidden ? kNegInf : x[k];
#pragma unroll
            for (int k = 0; k < 8; ++k) x[k] = ex2(x[k]);
            store_p(kC0 + i, pack_f16x2(x[0], x[1]), pack_f16x2(x[2], x[3]), pack_f16x2(x[4], x[5]), pack_f16x2(x[6], x[7]));
#pragma unroll
            for (int k = 0; k < 8; k += 2)
                f2_unpack(f2_add(f2_pack(l[i + k], l[i + k + 1]), f2_pack(x[k], x[k + 1])), l[i + k], l[i + k + 1]);
        }
        fence_async_smem();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&bars.p_full);
        if (warp == 4) {
            tc_wait(&bars.p_full, ph, dead, p.status);
            tc_fence_after();
            __syncwarp();
            if (alive(dead) && elect_one()) {
                tc_mma_values<kN>(tmem + F::kColO, smem, 0, kN, !starts);
                tc_commit(&bars.o_done);
            }
            __syncwarp();
        }
        if (!last) {
            advance(cur, s_len, nb, p.n_spans, kTcTile);
            continue;
        }
        // ---- the end of a piece: sums over the keys, then a dim a thread
        const bool whole = piece_t0 == 0 && cur.t + 1 == cur.T;
        const int out_slot = 2 * cta + (first_piece ? 0 : 1);
        float* s_sum = reinterpret_cast<float*>(s_red);
#pragma unroll
        for (int i = 0; i < kH; ++i) {
            if (!mine(i)) continue;
#pragma unroll
            for (int off = 16; off > 0; off >>= 1) l[i] += __shfl_xor_sync(0xffffffffu, l[i], off);
            if (lane == 0) s_sum[quad * kN + kC0 + i] = l[i];
        }
        workers_sync();
        if (key < n_cols) {
            const int row = kC0 + key;
            float sum = 0.f;
            for (int k = 0; k < 4; ++k) sum += s_sum[k * kN + row] + s_faint[k * kN + row];
            s_inv[row] = sum > 0.f ? (p.v_head ? __ldcg(p.v_head + head) : 1.f) / sum : sum == 0.f ? 0.f : sum;
            if (!whole && row < n_live) p.part_ml[(size_t)out_slot * p.n_rows + row] = make_float2(s_m[row], sum);
        }
        tc_wait(&bars.o_done, ph, dead, p.status);
        tc_fence_after();
        workers_sync();   // (s_inv)
        // row (i, g) of the span lies i Hq + g rows past its first one
        __nv_bfloat16* const dst = p.out + ((size_t)bg * p.R * p.Hq + (size_t)head * p.G + row0) * kPackDim + key;
        float* const part = p.part_o + (size_t)out_slot * p.n_rows * kPackDim + key;
#pragma unroll 1
        for (int i = 0; i < n_cols; i += 8) {
            float o[8];
            tc_ld8(tmem + lanes + F::kColO + kC0 + i, o);
            tc_wait_ld();
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const int row = kC0 + i + k;
                if (row >= n_live) continue;
                const float v = o[k] * s_inv[row];
                if (whole) dst[(s_draft[row0 + row] * (p.Hq - p.G) + row) * kPackDim] = __float2bfloat16(v);
                else part[row * kPackDim] = v;
            }
        }
        if (threadIdx.x == 0 && !whole && piece_t0 == 0) {
            const long long U = *reinterpret_cast<const long long*>(s_info + 2);
            const int Gc = s_info[4];
            const int n = cur.t + 1;   // the piece's tiles (it starts the span)
            const long long end = first_unit(cta + 1, U, Gc) - 1 + (cur.T - n);
            p.jobs[cta] = Job{bg, cur.h, out_slot, owner_of(end, U, Gc) - cta + 1};
        }
        tc_fence_before();
        first_piece = false;
        advance(cur, s_len, nb, p.n_spans, kTcTile);
        workers_sync();   // (the columns' words are free)
    }
    cp_async_wait<0>();
}

template <int kN>
__global__ void __launch_bounds__(kTcThreads, TcForm<kN>::kMinBlocks) packed_attention_tc_kernel(const PackedAttnParams p) {
    using F = TcForm<kN>;
    extern __shared__ uint4 smem_raw[];
    uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    __shared__ TcBars bars;
    __shared__ long long s_wsum[kTcThreads / 32];
    __shared__ alignas(16) int s_info[8];      // [2], [3] U; [4] the CTAs
    __shared__ uint32_t s_tmem;
    __shared__ volatile int s_dead;
    __shared__ int s_draft[2 * kTcMaxRows];   // of the KV head's query rows
    int* s_len = reinterpret_cast<int*>(smem + F::kOffLen);
    long long* s_prefix = reinterpret_cast<long long*>(smem);
    const int warp = threadIdx.x >> 5, cta = blockIdx.x, grid = gridDim.x;
    const int nb = p.n_batch;
    if (threadIdx.x == 0) {
        s_dead = 0;
        mbar_init(&bars.k_full, 4);
        mbar_init(&bars.s_full, 1);
        mbar_init(&bars.p_full, 8);
        mbar_init(&bars.o_done, 1);
        mbar_init(&bars.f_done, 1);
        fence_barrier_init();
    }
    for (int row = threadIdx.x; row < 2 * kTcMaxRows; row += kTcThreads) s_draft[row] = row / p.G;
    wait_prior_grid();
    allow_dependent_launch();
    const long long W = build_prefix<kTcThreads>(p, kTcTile, s_len, s_prefix, s_wsum);
    const bool few = W <= grid;
    const int X = few ? 0 : p.span_x, Gc = few ? (int)W : grid;
    if (threadIdx.x == 0) {
        p.jobs[cta].n = 0;
        if (cta == 0 && p.b_base == 0) *p.status = 0;
    }
    if (cta >= Gc) return;
    if (X > 0) {
        for (int b = threadIdx.x; b < nb; b += kTcThreads) s_prefix[b] += (long long)X * p.n_spans * b;
        __syncthreads();
    }
    const long long U = W + (long long)X * p.n_spans * nb;
    const Share share = share_of(cta, U, Gc, s_prefix, s_len, nb, p.n_spans, X, kTcTile);
    const int n_tiles = share.n_tiles;
    if (n_tiles <= 0) return;
    if (threadIdx.x == 0) {
        *reinterpret_cast<long long*>(s_info + 2) = U;
        s_info[4] = Gc;
    }
    if (warp == 0) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&s_tmem)),
                     "n"(F::kCols)
                     : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();   // the prefix gives way to V
    tc_fence_after();
    const uint32_t tmem = s_tmem;

    tc_worker<kN>(p, smem, bars, tmem, &s_dead, s_info, s_len, share.first, n_tiles, s_draft);
    // every MMA completes before the tensor memory is given back
    if (warp == 0 && !mbar_wait_bounded(&bars.o_done, (uint32_t)(n_tiles - 1) & 1) && threadIdx.x == 0)
        atomicOr(p.status, CS_DEVICE_WAIT_TIMEOUT);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (warp == 0)
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "n"(F::kCols) : "memory");
}
