// packed_attention_tc.cuh -- the tcgen05 form of packed attention, for 25 to 80
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
// One CTA an SM, every one of its buffers twice, so that the stages of a tile
// overlap those of the tiles beside it, each with warps of its own: K rows are
// decoded, V rows are, the softmax is done, and two warps issue the products for S
// and for O (an issue takes as long as its product).  The codes of the next two
// tiles come by cp.async meanwhile, every warp's own rows.  Scores are read as the
// fragments that stmatrix writes, so that a thread needs the scales of a quarter of
// the columns.  The sums of P are products too, with a matrix of ones: sums in
// registers took the softmax warps' room.
//
// As in the other form P = 2^(s - m + 12), and the tile is taken the short way
// unless some weight would leave [2^-14, 2^15] (a vote of the softmax warps).  Then
// (mend) the columns' maxima are found, O is rescaled where one grows by more than
// 2^3, and weights below 2^-14 (faint) are taken 28 powers of two at a time by
// products of their own, which the softmax warps add to O.  Mending is rolled up, for
// the instruction cache's sake.
//
// What bounds it: the softmax warps, at some 2300 (48 columns) to 3200 cycles (80) a
// tile (one set of decoding warps takes 2400), where the SM's instructions alone would
// take 1100 to 1500: chains of waits (a try_wait that succeeds costs 160 cycles, a vote
// 60 and the warps' drift), shared-memory and conversion latencies; the tensor pipe is
// 23 to 30% busy, DRAM 21 to 27%.  Every warp has the same 96 registers (72 up to 48
// columns), also those that issue and watch.  64 requests of 4096 keys and 8 KV heads:
// 32 rows 138 us, 36 148; 32 requests: 56 rows 98, 72 111; 256 requests of up to 16384
// keys, 72 rows: 1.34 ms for 2.8 GB (the same attention over a bf16 cache: 1.72 ms for
// 10 GB).  A CTA that does everything in turn, two an SM, took 2.03 ms.
// A tile that is mended costs several times one that is not, and peaked scores mend
// most tiles: with scores of 3, 5 and 8 nats' deviation 36 rows (64 requests) take 0.79,
// 1.08 and 1.58 ms and 72 rows (32 requests) 0.64, 0.96 and 1.36; with one key 20, 40 and 60
// nats above the rest 0.76, 1.18 and 1.59, and 0.61, 0.97 and 1.33.  A piece's first tile is
// always mended (m starts at -inf).
//
// Every mbarrier wait is bounded; after one that gives up nothing waits or is
// issued any more, every warp still meets every block barrier, and the status
// word says so.  A warp that issues products waits for its own at its end, so that
// none is in flight when the tensor memory is given back (drain).

constexpr int kTcTile = 128;                       // keys of a tile: the MMAs' M (S) and K (O)
constexpr int kTcVBytes = kTcTile * 256;           // V of a tile in fp16
constexpr int kTcRowBytes = kTcTile * (kPackCodeBytes + kPackGroups);   // codes and scales of K or V of a tile
constexpr int kTcMaxRows = 80;                     // query rows of a span at most

template <int kN>
struct TcForm {
    // Warps: eight decoders a set, one set or (up to 48 columns, where they are what
    // takes longest: 36 rows 162 us with one set, 151 with two; 56 rows 99 and 108,
    // for want of registers) two in turn; eight for the softmax; two that issue, one
    // that watches.
    static constexpr int kSets = kN <= 48 ? 2 : 1;
    static constexpr int kSoft = 8 * kSets, kIssueS = kSoft + 8, kIssueO = kIssueS + 1, kWatch = kIssueS + 2;
    static constexpr int kThreads = (kWatch + 4) / 4 * 4 * 32;           // (registers are given to four warps at a time)
    static constexpr int kH = kN / 2;                                    // columns of four softmax warps
    static_assert(kH % 8 == 0, "chunks of eight columns");
    static constexpr int kAtoms = kN > 64 ? 2 : 1;                       // 64-column atoms of P
    static constexpr int kPGroup = kAtoms * 1024;                        // bytes of P for 8 keys
    static constexpr int kPBytes = kTcTile / 8 * kPGroup;
    static constexpr int kQHalf = kN * 128;                              // bytes of a dim half of Q
    // tensor memory: K twice, S twice, O, the sums of P, the product of faint weights
    static constexpr int kColK = 0, kColS = 128, kColO = kColS + 2 * kN, kColL = kColO + kN, kColF = kColL + kN, kCols = 512;
    static_assert(kColF + 64 <= kCols, "tensor memory");
    // V | P | Q | raw rows, all twice | ones | columns | lengths
    static constexpr int kOffP = 2 * kTcVBytes, kOffQ = kOffP + 2 * kPBytes, kOffRaw = kOffQ + 4 * kQHalf;
    static constexpr int kOffOnes = kOffRaw + 4 * kTcRowBytes, kOffCol = kOffOnes + 2048, kOffLen = kOffCol + kN * 4 * (6 + 8);
    static constexpr int kSmem = kOffLen + kMaxBatchPerLaunch * 4 + 1024;
    static_assert(kOffOnes % 1024 == 0 && kSmem + 2048 <= 232448, "shared memory");
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
// 8 columns of 16 lanes: a thread columns 2c and 2c + 1 (c = lane % 4) of lanes lane / 4
// and lane / 4 + 8 (complete after tc_wait_ld)
__device__ __forceinline__ void tc_ld16(uint32_t addr, float* v) {
    asm volatile("tcgen05.ld.sync.aligned.16x256b.x1.b32 {%0,%1,%2,%3}, [%4];"
                 : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3])
                 : "r"(addr));
}
// Four 8 x 8 matrices of 16-bit values from their fragments; `addr`: the lane's row.
__device__ __forceinline__ void store_matrices(uint32_t addr, uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
    asm volatile("stmatrix.sync.aligned.m8n8.x4.shared.b16 [%0], {%1,%2,%3,%4};" ::"r"(addr), "r"(a), "r"(b), "r"(c), "r"(d)
                 : "memory");
}
// (after tc_wait_ld: nothing that uses them is moved before it)
__device__ __forceinline__ void tc_loaded8(float* v) {
    asm volatile("" : "+f"(v[0]), "+f"(v[1]), "+f"(v[2]), "+f"(v[3]), "+f"(v[4]), "+f"(v[5]), "+f"(v[6]), "+f"(v[7]));
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
// kind::f16, both operands fp16, fp32 sums, M = m, N = n
__host__ __device__ constexpr uint32_t tc_idesc(int m, int n, bool a_mn, bool b_mn) {
    return (1u << 4) | (a_mn ? 1u << 15 : 0u) | (b_mn ? 1u << 16 : 0u) | ((uint32_t)(n >> 3) << 17) | ((uint32_t)(m >> 4) << 24);
}

// Whether any of the softmax warps' threads says so; a barrier of theirs.
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
// The same, and with the watching warp.
__device__ __forceinline__ bool vote(bool x) {
    uint32_t r;
    asm volatile(
        "{\n\t.reg .pred p, q;\n\tsetp.ne.u32 p, %1, 0;\n\tbarrier.cta.red.or.pred q, 2, 288, p;\n\t"
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

// Tile j uses those of j % 2, whose phase j / 2 is its own.
struct TcBars {
    uint64_t q_full[2];    // Q of a piece written (4 warps)
    uint64_t k_full[2];    // K of a tile decoded (4 warps)
    uint64_t v_full[2];    // V of a tile decoded (4 warps)
    uint64_t s_full[2];    // S of a tile done; its K is read
    uint64_t p_full[2];    // P of a tile written, its S read (8 warps)
    uint64_t o_done[2];    // O of a tile done; its P and V are read
    uint64_t f_done;       // a product of faint weights done
    uint64_t drained[3];   // a warp's products done, at its end: one phase each
    int starts[2];         // whether a tile's products start O (1) and the sums (2); written before p_full
};

// The end of a warp that issued products: all of them are done, or a second has
// passed.  (On a barrier of a single phase: where a wait gave up, those of the buffers
// may be a phase behind, which a parity does not tell.)
__device__ __forceinline__ void tc_drain(uint64_t* drained, int* status) {
    if (elect_one()) tc_commit(drained);
    __syncwarp();
    if (!mbar_wait_bounded(drained, 0) && elect_one()) atomicOr(status, CS_DEVICE_WAIT_TIMEOUT);
}

// V^T P^T, n columns of P from an atom's first on, into the columns from d on
// (one thread issues): 8 steps of 16 keys.
template <int kN>
__device__ __forceinline__ void tc_mma_values(uint32_t d, uint8_t* smem, int buffer, int atom, int n, bool add) {
    using F = TcForm<kN>;
    const uint32_t id = tc_idesc(128, n, true, true);
    const uint64_t v = tc_desc(smem_u32(smem + buffer * kTcVBytes), 2048, 1024);
    const uint64_t x = tc_desc(smem_u32(smem + F::kOffP + buffer * F::kPBytes + atom * 1024), F::kPGroup, 1024);
#pragma unroll
    for (int kk = 0; kk < kTcTile / 16; ++kk)
        tc_mma_ss(d, v + (uint64_t)(kk * (4096 >> 4)), x + (uint64_t)(kk * 2 * F::kPGroup >> 4), id, add || kk > 0 ? 1u : 0u);
}

// The sums of P over the keys: 64 equal rows of ones times P, n columns.
template <int kN>
__device__ __forceinline__ void tc_mma_sums(uint32_t d, uint8_t* smem, int buffer, bool add) {
    using F = TcForm<kN>;
    const uint32_t id = tc_idesc(64, kN, true, true);
    const uint64_t ones = tc_desc(smem_u32(smem + F::kOffOnes), 1024, 1024);
    const uint64_t x = tc_desc(smem_u32(smem + F::kOffP + buffer * F::kPBytes), F::kPGroup, 1024);
#pragma unroll
    for (int kk = 0; kk < kTcTile / 16; ++kk)
        tc_mma_ss(d, ones, x + (uint64_t)(kk * 2 * F::kPGroup >> 4), id, add || kk > 0 ? 1u : 0u);
}

// Of the eight warps of a set the first four: K rows, and the query rows of a piece;
// the others: V rows.
template <int kN>
__device__ __forceinline__ void tc_decode(const PackedAttnParams& p, uint8_t* smem, TcBars& bars, uint32_t tmem,
                                          volatile int* dead, const int* s_len, const Cursor start, const int n_tiles,
                                          const int* s_draft) {
    using F = TcForm<kN>;
    const int warp = (threadIdx.x >> 5) & 7, lane = threadIdx.x & 31, quad = warp & 3, set = threadIdx.x >> 8;
    const bool v_side = warp >= 4;   // (one body of code for both: the instruction cache is small)
    const int key = 32 * quad + lane;                    // of a tile; also the lane of tensor memory
    const uint32_t lanes = (uint32_t)(32 * quad) << 16;
    const int nb = p.n_batch;
    float* s_sc = reinterpret_cast<float*>(smem + F::kOffCol);   // [2][N] scale of a column's scores

    // ---- the rows of the next two tiles: codes and scales into shared memory (parts
    // of the codes exchanged by the key's bits, so that the threads' 16-byte loads meet
    // every bank once)
    const uint8_t* codes = v_side ? p.v_codes : p.k_codes;
    const uint8_t* scales = v_side ? p.v_scales : p.k_scales;
    uint8_t* const raw = smem + F::kOffRaw + (v_side ? 2 * kTcRowBytes : 0);
    const int raw_x = (key >> 1) & 3;
    Cursor cl = start, cur = start;   // the tile whose page is looked up next, and tile j
    int next = set, piece = 0;        // cl's tile, j's piece
    for (int i = 0; i < set; ++i) {
        advance(cl, s_len, nb, p.n_spans, kTcTile);
        advance(cur, s_len, nb, p.n_spans, kTcTile);
        piece += cur.t == 0;
    }
    int page = -1, slot = 0;     // of the tile whose row is loaded next
    const int page_rows = p.Hkv * p.ps;
    auto look_up = [&]() {
        page = -1;
        if (next >= n_tiles) return;
        next += F::kSets;
        const int pos = cl.t * kTcTile + key;
        slot = (p.n_rb == 1 ? cl.h : cl.h / p.n_rb) * p.ps + (pos & (p.ps - 1));
        if (pos < s_len[cl.b])
            page = __ldcg(p.page_table + (size_t)(p.b_base + cl.b) * p.max_pages + (pos >> p.ps_log2));
        for (int i = 0; i < F::kSets; ++i) advance(cl, s_len, nb, p.n_spans, kTcTile);
    };
    auto load_rows = [&](int buffer) {   // zeros for a key past the context or on no page
        const int row = page >= 0 && page < p.P ? page * page_rows + slot : -1;
        uint8_t* const to = raw + buffer * kTcRowBytes;
#pragma unroll
        for (int i = 0; i < 4; ++i) {    // four lanes a row: keys of a page lie side by side
            const int of = 8 * i + (lane >> 2), r = __shfl_sync(0xffffffffu, row, of);
            cp_async16(smem_u32(to + (32 * quad + of) * kPackCodeBytes + (((lane & 3) ^ (of >> 1 & 3)) << 4)),
                       codes + (size_t)max(r, 0) * kPackCodeBytes + 16 * (lane & 3), r >= 0);
        }
        cp_async8(smem_u32(to + kTcTile * kPackCodeBytes + key * kPackGroups), scales + (size_t)max(row, 0) * kPackGroups,
                  row >= 0);
        cp_async_commit();
        look_up();
    };
    // a row as fp16, into tensor memory (K) or shared memory (V)
    auto decode = [&](int buffer) {
        const uint8_t* const from = raw + buffer * kTcRowBytes;
        const uint2 sc8 = *reinterpret_cast<const uint2*>(from + kTcTile * kPackCodeBytes + key * kPackGroups);
        uint8_t* const v_row = smem + buffer * kTcVBytes + (key >> 3) * 2048 + (key & 7) * 128;
        uint4 all[4];   // (requested together: no load is moved before a store below)
#pragma unroll
        for (int i = 0; i < 4; ++i)
            all[i] = *reinterpret_cast<const uint4*>(from + key * kPackCodeBytes + ((i ^ raw_x) << 4));
#pragma unroll
        for (int i = 0; i < 4; ++i) {   // 32 dims: 16 pairs
            const uint32_t w[4] = {all[i].x, all[i].y, all[i].z, all[i].w};
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
                tc_st16(tmem + lanes + F::kColK + buffer * 64 + 16 * i, x);
            } else {
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    *reinterpret_cast<uint4*>(v_row + (i >> 1) * 1024 + ((((i & 1) * 4 + j) ^ (key & 7)) << 4)) =
                        make_uint4(x[4 * j], x[4 * j + 1], x[4 * j + 2], x[4 * j + 3]);
            }
        }
    };
    look_up();
    load_rows(set);
    if (F::kSets == 1) load_rows(1);
#pragma unroll 1
    for (int j = set; j < n_tiles; j += F::kSets) {
        const int buf = j & 1;
        const uint32_t ph = (uint32_t)(j >> 1) & 1;
        // ---- what was in the place of this tile's row is read
        if (j >= 2) tc_wait(v_side ? &bars.o_done[buf] : &bars.s_full[buf], ph ^ 1, dead, p.status);
        tc_fence_after();
        if (!v_side && (j == 0 || cur.t == 0)) {
            // ---- a new piece: its query rows as fp16 below 2^15 (as in the other form),
            // a lane its four dims of a row, converted where they arrive.  (Their buffer was
            // read last by the tile two before, or an earlier one.  This wait is right only
            // after the one above: S of that tile is issued after P of the tile two before it,
            // and a parity does not tell a phase from the one two before.)
            if (j >= 2) tc_wait(&bars.p_full[buf], ph ^ 1, dead, p.status);
            // the KV head of the span, and its row block's first row
            const int bg = p.b_base + cur.b;
            const int head = p.n_rb == 1 ? cur.h : cur.h / p.n_rb, row0 = (cur.h - head * p.n_rb) * p.n_rows;
            const int n_live = min(p.n_rows, p.n_all - row0);
            uint8_t* const s_q = smem + F::kOffQ + (piece & 1) * 2 * F::kQHalf + (lane >> 4) * F::kQHalf + (lane & 1) * 8;
            const float scale = p.scale_log2 * (p.k_head ? __ldcg(p.k_head + head) : 1.f);
            const __nv_bfloat16* const from =
                p.q + ((size_t)bg * p.R * p.Hq + (size_t)head * p.G + row0) * kPackDim + 4 * lane;
            auto place = [&](int row) { return s_q + row * 128 + ((((lane & 15) >> 1) ^ (row & 7)) << 4); };
#pragma unroll 4
            for (int row = warp; row < kN; row += 4) {
                const bool in = row < n_live;   // row (i, g) lies i Hq + g rows past its head's first one
                const __nv_bfloat16* src = from + (in ? (size_t)(s_draft[row0 + row] * (p.Hq - p.G) + row) * kPackDim : 0);
                const uint32_t to = smem_u32(place(row));
                cp_async4(to, src, in);
                cp_async4(to + 4, src + 2, in);
            }
            cp_async_commit();
            cp_async_wait<0>();
#pragma unroll 4
            for (int row = warp; row < kN; row += 4) {
                float back;
                uint2* const at = reinterpret_cast<uint2*>(place(row));
                *at = query_f16(*at, back);
                // (not 0, under which a hidden score would be NaN)
                if (lane == 0) s_sc[(piece & 1) * kN + row] = row < n_live ? fmaxf(scale * back, 0x1p-126f) : 0x1p-126f;
            }
            fence_async_smem();
            __syncwarp();
            if (lane == 0) mbar_arrive(&bars.q_full[piece & 1]);
        }
        // ---- this tile's row, and the request of that two tiles on
        cp_async_wait<2 - F::kSets>();
        __syncwarp();
        decode(buf);
        __syncwarp();
        load_rows(buf);
        if (v_side) {
            fence_async_smem();
            __syncwarp();
            if (lane == 0) mbar_arrive(&bars.v_full[buf]);
        } else {
            tc_wait_st();
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(&bars.k_full[buf]);
        }
        for (int i = 0; i < F::kSets; ++i) {
            advance(cur, s_len, nb, p.n_spans, kTcTile);
            piece += cur.t == 0;
        }
    }
    cp_async_wait<0>();
}

// A warp: the products for S.
template <int kN>
__device__ __forceinline__ void tc_issue_scores(const PackedAttnParams& p, uint8_t* smem, TcBars& bars, uint32_t tmem,
                                                volatile int* dead, const int* s_len, const Cursor start, const int n_tiles) {
    using F = TcForm<kN>;
    Cursor cur = start;
    int piece = -1;
#pragma unroll 1
    for (int j = 0; j < n_tiles; ++j) {
        const int buf = j & 1;
        const uint32_t ph = (uint32_t)(j >> 1) & 1;
        if (j == 0 || cur.t == 0) ++piece;
        tc_wait(&bars.k_full[buf], ph, dead, p.status);
        if (j >= 2) tc_wait(&bars.p_full[buf], ph ^ 1, dead, p.status);
        tc_fence_after();
        __syncwarp();
        if (alive(dead) && elect_one()) {
            const uint64_t dq = tc_desc(smem_u32(smem + F::kOffQ + (piece & 1) * 2 * F::kQHalf), 1024, 0);
#pragma unroll
            for (int ks = 0; ks < kPackDim / 16; ++ks)
                tc_mma_ts(tmem + F::kColS + buf * kN, tmem + F::kColK + buf * 64 + ks * 8,
                          dq + (uint64_t)((ks >> 2) * (F::kQHalf >> 4) + (ks & 3) * 2), tc_idesc(128, kN, false, false),
                          ks > 0 ? 1u : 0u);
            tc_commit(&bars.s_full[buf]);
        }
        __syncwarp();
        advance(cur, s_len, p.n_batch, p.n_spans, kTcTile);
    }
    tc_drain(&bars.drained[0], p.status);
}

// A warp: the products for O and the sums.
template <int kN>
__device__ __forceinline__ void tc_issue_values(const PackedAttnParams& p, uint8_t* smem, TcBars& bars, uint32_t tmem,
                                                volatile int* dead, const int n_tiles) {
    using F = TcForm<kN>;
#pragma unroll 1
    for (int j = 0; j < n_tiles; ++j) {
        const int buf = j & 1;
        const uint32_t ph = (uint32_t)(j >> 1) & 1;
        tc_wait(&bars.v_full[buf], ph, dead, p.status);
        tc_wait(&bars.p_full[buf], ph, dead, p.status);
        tc_fence_after();
        const int starts = *reinterpret_cast<volatile int*>(&bars.starts[buf]);
        __syncwarp();
        if (alive(dead) && elect_one()) {
            tc_mma_values<kN>(tmem + F::kColO, smem, buf, 0, kN, !(starts & 1));
            tc_mma_sums<kN>(tmem + F::kColL, smem, buf, !(starts & 2));
            tc_commit(&bars.o_done[buf]);
        }
        __syncwarp();
    }
    tc_drain(&bars.drained[1], p.status);
}

// A warp: takes part in a tile's vote once the place of its P is free, so that the
// softmax warps do not each look.
__device__ __forceinline__ void tc_watch(const PackedAttnParams& p, TcBars& bars, volatile int* dead, const int n_tiles) {
#pragma unroll 1
    for (int j = 0; j < n_tiles; ++j) {
        if (j >= 2) tc_wait(&bars.o_done[j & 1], (uint32_t)((j >> 1) & 1) ^ 1, dead, p.status);
        __syncwarp();
        vote(false);
    }
}

// The softmax and the results.
template <int kN>
__device__ __forceinline__ void tc_softmax(const PackedAttnParams& p, uint8_t* smem, TcBars& bars, uint32_t tmem,
                                           volatile int* dead, const int* s_info, const int* s_len, const Cursor start,
                                           const int n_tiles, const int* s_draft) {
    using F = TcForm<kN>;
    constexpr int kH = F::kH;
    const int warp = (threadIdx.x >> 5) - F::kSoft, lane = threadIdx.x & 31, quad = warp & 3;
    const int kC0 = warp >= 4 ? kH : 0;                  // this warp's columns
    constexpr int n_cols = kH;
    const int key = 32 * quad + lane;                    // of a tile; also the lane of tensor memory
    const uint32_t lanes = (uint32_t)(32 * quad) << 16;
    const int nb = p.n_batch, cta = blockIdx.x;
    float* s_sc = reinterpret_cast<float*>(smem + F::kOffCol);   // [N] scale of a column's scores (of two pieces)
    float* s_up = s_sc + 2 * kN;                         // [N] 12 - m
    float* s_alpha = s_up + kN;                          // [N] what a column's sums are rescaled by
    float* s_m = s_alpha + kN;                           // [N] running maxima
    float* s_inv = s_m + kN;                             // [N] 1 / l at the end
    int* s_red = reinterpret_cast<int*>(s_inv + kN);     // [4][N] the quads' maxima, or sums
    float* s_faint = reinterpret_cast<float*>(s_red + 4 * kN);   // [4][N] the quads' sums of faint weights
    const uint32_t o_at = tmem + lanes + F::kColO + kC0, l_at = tmem + lanes + F::kColL + kC0;

    // eight of a key's columns of P, from `col` on
    auto store_p = [&](int buf, int col, uint32_t x0, uint32_t x1, uint32_t x2, uint32_t x3) {
        uint8_t* const p_row = smem + F::kOffP + buf * F::kPBytes + (key >> 3) * F::kPGroup + (key & 7) * 128;
        *reinterpret_cast<uint4*>(p_row + (col >> 6) * 1024 + ((((col & 63) >> 3) ^ (key & 7)) << 4)) =
            make_uint4(x0, x1, x2, x3);
    };
    Cursor cur = start;
    bool first_piece = true;
    uint32_t f_phase = 0;
    int piece_t0 = cur.t, piece = 0;
    int L = 0, bg = 0, head = 0, row0 = 0, n_live = 0, left = 0;   // of the piece; its tiles from the next on
#pragma unroll 1
    for (int j = 0; j < n_tiles; ++j) {
        const int buf = j & 1;
        const uint32_t ph = (uint32_t)(j >> 1) & 1;
        const bool first = left == 0;
        if (first) {
            piece_t0 = cur.t;
            left = min(cur.T - cur.t, n_tiles - j);
            L = s_len[cur.b];
            bg = p.b_base + cur.b;
            head = p.n_rb == 1 ? cur.h : cur.h / p.n_rb;
            row0 = (cur.h - head * p.n_rb) * p.n_rows;
            n_live = min(p.n_rows, p.n_all - row0);
            const int row = threadIdx.x - 32 * F::kSoft;
            if (row < kN) {
                s_up[row] = row < n_live ? -kNegInf : 0.f;
                s_m[row] = row < n_live ? kNegInf : kPUp;
                for (int k4 = 0; k4 < 4; ++k4) s_faint[k4 * kN + row] = 0.f;
            }
            tc_wait(&bars.q_full[piece & 1], (uint32_t)(piece >> 1) & 1, dead, p.status);
            s_sc = reinterpret_cast<float*>(smem + F::kOffCol) + (piece & 1) * kN;
            ++piece;
            workers_sync();
        }
        // ---- softmax: this key's scores
        tc_wait(&bars.s_full[buf], ph, dead, p.status);
        tc_fence_after();
        const uint32_t s_at = tmem + lanes + F::kColS + buf * kN + kC0;
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
                tc_loaded8(z);
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
            auto is_faint = [&](float x) { return x < kPMin && x > kPGone; };
            bool faint = false;
#pragma unroll 1
            for (int i = 0; i < n_cols; i += 8) {
                float z[8];
                tc_ld8(s_at + i, z);
                tc_wait_ld();
                tc_loaded8(z);
#pragma unroll
                for (int k = 0; k < 8; ++k)
                    faint |= kC0 + i + k >= hidden && is_faint(fmaf(z[k], s_sc[kC0 + i + k], s_up[kC0 + i + k]));
            }
            faint = workers_any(faint);
            if ((rescale || faint) && !first) {
                tc_wait(&bars.o_done[buf ^ 1], (uint32_t)((j - 1) >> 1) & 1, dead, p.status);
                tc_fence_after();
            }
            if (rescale) {
#pragma unroll 1
                for (int i = 0; i < (quad == 0 ? 2 : 1) * n_cols; i += 8) {   // (the sums: in the first quad's lanes)
                    const int col = i < n_cols ? i : i - n_cols;
                    const uint32_t at = (i < n_cols ? o_at : l_at) + col;
                    float o[8];
                    tc_ld8(at, o);
                    tc_wait_ld();
                    tc_loaded8(o);
#pragma unroll
                    for (int k = 0; k < 8; ++k) o[k] *= s_alpha[kC0 + col + k];
                    tc_st8(at, reinterpret_cast<const uint32_t*>(o));
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
                    tc_loaded8(z);
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
                    store_p(buf, kC0 + i, pack_f16x2(f[0], f[1]), pack_f16x2(f[2], f[3]), pack_f16x2(f[4], f[5]),
                            pack_f16x2(f[6], f[7]));
                }
                tc_wait_st();
                fence_async_smem();
                const float down = ex2(-up);
#pragma unroll 1
                for (int atom = 0; atom < F::kAtoms; ++atom) {   // 64 columns at a time
                    tc_fence_before();
                    workers_sync();
                    tc_fence_after();
                    if (warp == 0) {
                        tc_wait(&bars.v_full[buf], ph, dead, p.status);
                        __syncwarp();
                        if (alive(dead) && elect_one()) {
                            tc_mma_values<kN>(tmem + F::kColF, smem, buf, atom, min(64, kN - 64 * atom), false);
                            tc_commit(&bars.f_done);
                        }
                        __syncwarp();
                    }
                    tc_wait(&bars.f_done, f_phase, dead, p.status);
                    f_phase ^= 1;
                    tc_fence_after();
#pragma unroll 1
                    for (int i = 0; i < n_cols; i += 8) {
                        if ((kC0 + i) >> 6 != atom) continue;
                        float o[8], f[8];
                        tc_ld8(tmem + lanes + F::kColF + ((kC0 + i) & 63), f);
                        tc_ld8(o_at + i, o);
                        tc_wait_ld();
                        tc_loaded8(f);
                        tc_loaded8(o);
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
        // x = s - m + 12 of this warp's columns: eight of a chunk c, columns col(c) and
        // col(c) + 1 of the keys row(0) .. row(3) of the warp's 32
        float x[kH];
        auto col = [&](int c) { return kC0 + 8 * c + 2 * (lane & 3); };
        auto row = [&](int h) { return 8 * h + (lane >> 2); };
        auto scores = [&]() {
#pragma unroll
            for (int c = 0; c < kH / 8; ++c) {
                tc_ld16(s_at + 8 * c, x + 8 * c);
                tc_ld16(s_at + (16u << 16) + 8 * c, x + 8 * c + 4);
            }
            tc_wait_ld();
#pragma unroll
            for (int c = 0; c < kH / 8; ++c) {
                tc_loaded8(x + 8 * c);
                const float2 m = *reinterpret_cast<const float2*>(s_sc + col(c)), u = *reinterpret_cast<const float2*>(s_up + col(c));
#pragma unroll
                for (int k = 8 * c; k < 8 * c + 8; k += 2)
                    f2_unpack(f2_fma(f2_pack(x[k], x[k + 1]), f2_pack(m.x, m.y), f2_pack(u.x, u.y)), x[k], x[k + 1]);
            }
        };
        // what is hidden becomes `with`
        auto hide = [&](float with) {
#pragma unroll
            for (int h = 0; h < 4; ++h) {
                const int of = key0 + 32 * quad + row(h);
                const int none = of >= L ? kN : (of - (L - p.R)) * p.G - row0;   // columns below it
#pragma unroll
                for (int c = 0; c < kH / 8; ++c)
#pragma unroll
                    for (int k = 0; k < 2; ++k) x[8 * c + 2 * h + k] = col(c) + k < none ? with : x[8 * c + 2 * h + k];
            }
        };
        scores();
        if (edge) hide(0.f);
        float most = 0.f, least = 0.f;
#pragma unroll
        for (int i = 0; i < kH; i += 2) {
            most = fmax3(most, x[i], x[i + 1]);
            least = fmin3(least, x[i], x[i + 1]);
        }
        const bool bad = vote(most > kPMax || least < kPMin);   // (P is free, too)
        if (bad) {
            mend();
            scores();
        }
        if (edge) hide(kNegInf);
        const uint32_t p_row = smem_u32(smem + F::kOffP + buf * F::kPBytes + (key >> 3) * F::kPGroup + (key & 7) * 128);
#pragma unroll
        for (int c = 0; c < kH / 8; ++c) {
            uint32_t f[4];
#pragma unroll
            for (int h = 0; h < 4; ++h) f[h] = pack_f16x2(ex2(x[8 * c + 2 * h]), ex2(x[8 * c + 2 * h + 1]));
            const int at = kC0 + 8 * c;
            store_matrices(p_row + (at >> 6) * 1024 + ((((at & 63) >> 3) ^ (key & 7)) << 4), f[0], f[1], f[2], f[3]);
        }
        fence_async_smem();
        tc_fence_before();
        if (threadIdx.x == 32 * F::kSoft) bars.starts[buf] = (starts ? 1 : 0) | (first ? 2 : 0);
        __syncwarp();
        if (lane == 0) mbar_arrive(&bars.p_full[buf]);
        if (--left > 0) {
            ++cur.t;
            continue;
        }
        // ---- the end of a piece: a dim a thread
        const bool whole = piece_t0 == 0 && cur.t + 1 == cur.T;
        const int out_slot = 2 * cta + (first_piece ? 0 : 1);
        float* s_sum = reinterpret_cast<float*>(s_red);
        tc_wait(&bars.o_done[buf], ph, dead, p.status);
        tc_fence_after();
        if (quad == 0) {
#pragma unroll 1
            for (int i = 0; i < n_cols; i += 8) {
                float o[8];
                tc_ld8(l_at + i, o);
                tc_wait_ld();
                tc_loaded8(o);
                if (lane == 0) {
                    *reinterpret_cast<float4*>(s_sum + kC0 + i) = make_float4(o[0], o[1], o[2], o[3]);
                    *reinterpret_cast<float4*>(s_sum + kC0 + i + 4) = make_float4(o[4], o[5], o[6], o[7]);
                }
            }
        }
        workers_sync();
        if (key < n_cols) {
            const int row = kC0 + key;
            float sum = s_sum[row];
            for (int k = 0; k < 4; ++k) sum += s_faint[k * kN + row];
            s_inv[row] = sum > 0.f ? (p.v_head ? __ldcg(p.v_head + head) : 1.f) / sum : sum == 0.f ? 0.f : sum;
            if (!whole && row < n_live) p.part_ml[(size_t)out_slot * p.n_rows + row] = make_float2(s_m[row], sum);
        }
        workers_sync();   // (s_inv)
        // row (i, g) of the span lies i Hq + g rows past its first one
        __nv_bfloat16* const dst = p.out + ((size_t)bg * p.R * p.Hq + (size_t)head * p.G + row0) * kPackDim + key;
        float* const part = p.part_o + (size_t)out_slot * p.n_rows * kPackDim + key;
#pragma unroll 1
        for (int i = 0; i < n_cols; i += 8) {
            float o[8];
            tc_ld8(o_at + i, o);
            tc_wait_ld();
            tc_loaded8(o);
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const int row = kC0 + i + k;
                if (row >= n_live) continue;
                const float v = o[k] * s_inv[row];
                if (whole) dst[(size_t)(s_draft[row0 + row] * (p.Hq - p.G) + row) * kPackDim] = __float2bfloat16(v);
                else part[row * kPackDim] = v;
            }
        }
        if (threadIdx.x == 32 * F::kSoft && !whole && piece_t0 == 0) {
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
    // (faint weights' products are waited for one by one, unless a wait gave up)
    if (warp == 0 && !alive(dead)) tc_drain(&bars.drained[2], p.status);
}

template <int kN>
__global__ void __launch_bounds__(TcForm<kN>::kThreads, 1) packed_attention_tc_kernel(const PackedAttnParams p) {
    using F = TcForm<kN>;
    extern __shared__ uint4 smem_raw[];
    uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    __shared__ TcBars bars;
    __shared__ long long s_wsum[F::kThreads / 32];
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
        for (int i = 0; i < 2; ++i) {
            mbar_init(&bars.q_full[i], 4);
            mbar_init(&bars.k_full[i], 4);
            mbar_init(&bars.v_full[i], 4);
            mbar_init(&bars.s_full[i], 1);
            mbar_init(&bars.p_full[i], 8);
            mbar_init(&bars.o_done[i], 1);
        }
        mbar_init(&bars.f_done, 1);
        for (int i = 0; i < 3; ++i) mbar_init(&bars.drained[i], 1);
        fence_barrier_init();
    }
    for (int row = threadIdx.x; row < 2 * kTcMaxRows; row += F::kThreads) s_draft[row] = row / p.G;
    wait_prior_grid();
    allow_dependent_launch();
    const long long W = build_prefix<F::kThreads>(p, kTcTile, s_len, s_prefix, s_wsum);
    const bool few = W <= grid;
    const int X = few ? 0 : p.span_x, Gc = few ? (int)W : grid;
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
    uint32_t* const ones = reinterpret_cast<uint32_t*>(smem + F::kOffOnes);
    if (threadIdx.x < 512) ones[threadIdx.x] = 0x3c003c00u;
    fence_async_smem();
    tc_fence_before();
    __syncthreads();   // the prefix gives way to V
    tc_fence_after();
    const uint32_t tmem = s_tmem;

    if (warp < F::kSoft) tc_decode<kN>(p, smem, bars, tmem, &s_dead, s_len, share.first, n_tiles, s_draft);
    else if (warp == F::kIssueS) tc_issue_scores<kN>(p, smem, bars, tmem, &s_dead, s_len, share.first, n_tiles);
    else if (warp == F::kIssueO) tc_issue_values<kN>(p, smem, bars, tmem, &s_dead, n_tiles);
    else if (warp == F::kWatch) tc_watch(p, bars, &s_dead, n_tiles);
    else if (warp < F::kIssueS) tc_softmax<kN>(p, smem, bars, tmem, &s_dead, s_info, s_len, share.first, n_tiles, s_draft);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (warp == 0)
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "n"(F::kCols) : "memory");
}
