// packed_attention_tc.cuh -- the tcgen05 form of packed attention, for 17 to 128
// query rows per KV head (included by packed_attention.cu inside its anonymous
// namespace: the same split of the keys, pieces and merge).
//
// Transposed products, so that the padding is to 16 query rows (N) and the keys
// and dims fill M = 128:
//   S^T [128 keys x N] = K Q^T    K as fp16 in tensor memory (a thread decodes
//       the row of its key, its lane), Q a K-major shared-memory operand;
//   O^T [128 dims x N] += V^T P^T  V as fp16 and P in shared memory, both
//       MN-major: a thread writes the row of its key as it is.
// What bounds it: shared memory.  A tile of 128 keys writes V (32 KB) and P and
// lets the tensor core read V, P and Q: with N = 80 some 1200 cycles at 128
// bytes, where 18 KB of codes take 800 at the memory's rate, the MMAs 640, the
// exponentials 640.  K goes by tensor memory, which takes it off that path.
//
// One CTA an SM of 17 warps.  Sixteen workers are four groups of four warps, a
// thread of a group one key of the tile: groups 0 and 2 decode the halves of
// its K row, groups 1 and 3 those of its V row, one tile ahead of the softmax,
// with the codes of the tile after that already requested into registers.  Then
// all do the softmax of the tile, each group a quarter of the columns (query
// rows).  (With eight warps, whole rows and half the columns each, a tile of 72
// rows took 3600 cycles, most of them waits on the warps' own results.)  Warp 16
// issues the MMAs: S of the next tile beside the softmax of this one, O of the
// last.
//
// As in the other form P = 2^(s - m + 12), and the tile is taken the short way
// unless some weight leaves [2^-14, 2^15] or some key is hidden from some row
// (a vote of the workers).  Then the columns' maxima are found, and O is
// rescaled where one grows by more than 2^3; weights below 2^-14 (faint) are
// taken 28 powers of two at a time by products of their own into the place of
// the tile's S, which the workers add to O.
//
// Every mbarrier wait is bounded; after one that gives up nothing waits or is
// issued any more, every warp still meets every block barrier, and the status
// word says so.

constexpr int kTcThreads = 544;
constexpr int kTcWorkers = 512;
constexpr int kTcTile = 128;                       // keys of a tile: the MMAs' M (S) and K (O)
constexpr int kTcVBytes = kTcTile * 256;           // V of a tile in fp16
constexpr int kTcVBufs = 3;
constexpr int kTcMinRows = 17, kTcMaxRows = 128;   // query rows that it takes

template <int kN>
struct TcForm {
    // columns of groups 0 and 1, and of groups 2 and 3: multiples of 8
    static constexpr int kH0 = (kN + 31) / 32 * 8, kH1 = kN / 2 - kH0;
    static constexpr int kNHalves = kN > 64 ? 2 : 1;                     // 64-column atoms of P
    static constexpr int kPGroup = kNHalves * 1024;                      // bytes of P for 8 keys
    static constexpr int kPBytes = kTcTile / 8 * kPGroup;
    static constexpr int kQHalf = kN * 128;                              // bytes of a dim half of Q
    static constexpr int kColS = 128, kColO = kColS + 2 * kN;            // tensor memory: K [0, 128), S twice, O
    static_assert(kColO + kN <= 512, "tensor memory");
    // V ring | P twice | Q | columns | lengths
    static constexpr int kOffP = kTcVBufs * kTcVBytes, kOffQ = kOffP + 2 * kPBytes, kOffCol = kOffQ + 2 * kQHalf;
    static constexpr int kOffLen = kOffCol + kN * 4 * (6 + 4);
    static constexpr int kSmem = kOffLen + kMaxBatchPerLaunch * 4 + 1024;
    static_assert(kSmem <= 232448 - 1024, "shared memory");
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

__device__ __forceinline__ void load32(const uint8_t* p, uint32_t* r) {   // 32 bytes, 32-byte aligned
    asm volatile("ld.global.cg.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7])
                 : "l"(p)
                 : "memory");
}
__device__ __forceinline__ uint32_t max_f16x2(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("max.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}
__device__ __forceinline__ uint32_t min_f16x2(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("min.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}
// Whether any of the workers' threads says so; a barrier of theirs.
__device__ __forceinline__ bool workers_any(bool x) {
    uint32_t r;
    asm volatile(
        "{\n\t.reg .pred p, q;\n\tsetp.ne.u32 p, %1, 0;\n\tbarrier.cta.red.or.pred q, 1, 512, p;\n\t"
        "selp.u32 %0, 1, 0, q;\n\t}\n"
        : "=r"(r)
        : "r"((uint32_t)x)
        : "memory");
    return r != 0;
}
__device__ __forceinline__ void workers_sync() { asm volatile("barrier.cta.sync 1, 512;" ::: "memory"); }

// A float's bits as an integer of the same order, and back.
__device__ __forceinline__ int ordered(float x) {
    const int b = __float_as_int(x);
    return b < 0 ? b ^ 0x7fffffff : b;
}
__device__ __forceinline__ float unordered(int b) { return __int_as_float(b < 0 ? b ^ 0x7fffffff : b); }

// Bounded; returns at once when another wait has given up.
__device__ __forceinline__ void tc_wait(uint64_t* bar, uint32_t parity, volatile int* dead, int* status) {
    if (mbar_test_wait(bar, parity) || *dead) return;
    if (mbar_wait_bounded(bar, parity)) return;
    *dead = 1;
    atomicOr(status, CS_DEVICE_WAIT_TIMEOUT);
}

// Whether no wait has given up, the same answer in the whole warp.
__device__ __forceinline__ bool alive(volatile int* dead) { return !__any_sync(0xffffffffu, *dead); }

struct TcBars {
    uint64_t k_full[2];    // K of a tile decoded (8 warps)
    uint64_t s_full[2];    // S of a tile done; its K is read
    uint64_t p_full[2];    // P and V of a tile written, its S read (16 warps)
    uint64_t o_done[2];    // O of a tile done; its P and V are read
    uint64_t f_done;       // a product of faint weights done
};

// V^T P^T of tile j into the columns from d on (one thread issues): 8 steps of 16 keys.
template <int kN>
__device__ __forceinline__ void tc_mma_values(uint32_t d, uint8_t* smem, int j, bool add) {
    using F = TcForm<kN>;
    constexpr uint32_t id = tc_idesc(kN, true, true);
    const uint64_t v = tc_desc(smem_u32(smem + (j % kTcVBufs) * kTcVBytes), 2048, 1024);
    const uint64_t x = tc_desc(smem_u32(smem + F::kOffP + (j & 1) * F::kPBytes), F::kPGroup, 1024);
#pragma unroll
    for (int kk = 0; kk < kTcTile / 16; ++kk)
        tc_mma_ss(d, v + (uint64_t)(kk * (4096 >> 4)), x + (uint64_t)(kk * 2 * F::kPGroup >> 4), id, add || kk > 0 ? 1u : 0u);
}

// kH columns from kC0 on; group: what of a row this warp decodes.
template <int kN, int kH>
__device__ __forceinline__ void tc_worker(const PackedAttnParams& p, uint8_t* smem, TcBars& bars, uint32_t tmem,
                                          volatile int* dead, int* s_info, const int* s_len, const Cursor start,
                                          const int n_tiles, const int* s_draft, const int kC0) {
    using F = TcForm<kN>;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, quad = warp & 3;
    const bool v_side = warp & 4;
    const int half = warp >> 3;                          // of the row: dims 64 half ..
    const int key = 32 * quad + lane;                    // of a tile; also the lane of tensor memory
    const uint32_t lanes = (uint32_t)(32 * quad) << 16;
    const int nb = p.n_batch, cta = blockIdx.x;
    float* s_sc = reinterpret_cast<float*>(smem + F::kOffCol);   // [N] scale of a column's scores
    float* s_up = s_sc + kN;                             // [N] 12 - m
    float* s_alpha = s_up + kN;                          // [N] what a column's sums are rescaled by
    float* s_m = s_alpha + kN;                           // [N] running maxima
    float* s_inv = s_m + kN;                             // [N] 1 / l at the end
    float* s_l = s_inv + kN;                             // [N]
    int* s_red = reinterpret_cast<int*>(s_l + kN);       // [4][N] the quads' maxima, or sums
    uint8_t* s_p = smem + F::kOffP;
    uint8_t* s_q = smem + F::kOffQ;

    // ---- the codes and scales of a tile's row, two tiles ahead
    const uint8_t* codes = (v_side ? p.v_codes : p.k_codes) + half * (kPackCodeBytes / 2);
    const uint8_t* scales = (v_side ? p.v_scales : p.k_scales) + half * (kPackGroups / 2);
    Cursor cl = start;           // the tile whose page is looked up next
    int left = n_tiles;
    int page = -1, slot = 0;     // of the tile whose row is loaded next
    uint32_t w[8], sc4 = 0;
    auto look_up = [&]() {
        page = -1;
        if (left <= 0) return;
        --left;
        const int pos = cl.t * kTcTile + key;
        slot = cl.h * p.ps + (pos & (p.ps - 1));
        if (pos < s_len[cl.b])
            page = __ldcg(p.page_table + (size_t)(p.b_base + cl.b) * p.max_pages + (pos >> p.ps_log2));
        advance(cl, s_len, nb, p.Hkv, kTcTile);
    };
    auto load_row = [&]() {      // zeros for a key past the context or on no page
        if (page >= 0 && page < p.P) {
            const size_t row = (size_t)page * p.Hkv * p.ps + slot;
            load32(codes + row * kPackCodeBytes, w);
            sc4 = __ldcg(reinterpret_cast<const uint32_t*>(scales + row * kPackGroups));
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) w[i] = 0;
            sc4 = 0;
        }
        look_up();
    };
    // half a row as fp16, into tensor memory (K) or shared memory (V)
    uint8_t* const v_row = smem + (key >> 3) * 2048 + half * 1024 + (key & 7) * 128;
    auto decode = [&](int tile) {
        const uint32_t f[2] = {scales_f16x2(sc4), scales_f16x2(sc4 >> 16)};
#pragma unroll
        for (int i = 0; i < 2; ++i) {   // 32 dims: 16 pairs
            uint32_t x[16];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const uint32_t s = __byte_perm(f[i], 0, j < 2 ? 0x1010 : 0x3232);
                x[4 * j] = mul_f16x2(codes_f16x2<0>(w[4 * i + j]), s);
                x[4 * j + 1] = mul_f16x2(codes_f16x2<1>(w[4 * i + j]), s);
                x[4 * j + 2] = mul_f16x2(codes_f16x2<2>(w[4 * i + j]), s);
                x[4 * j + 3] = mul_f16x2(codes_f16x2<3>(w[4 * i + j]), s);
            }
            if (!v_side) {
                tc_st16(tmem + lanes + (tile & 1) * 64 + half * 32 + 16 * i, x);
            } else {
                uint8_t* v = v_row + (tile % kTcVBufs) * kTcVBytes;
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    *reinterpret_cast<uint4*>(v + (((i * 4 + j) ^ (key & 7)) << 4)) =
                        make_uint4(x[4 * j], x[4 * j + 1], x[4 * j + 2], x[4 * j + 3]);
            }
        }
        if (!v_side) {
            tc_wait_st();
            tc_fence_before();
        } else {
            fence_async_smem();
        }
    };
    auto k_arrive = [&](int tile) {
        __syncwarp();
        if (!v_side && lane == 0) mbar_arrive(&bars.k_full[tile & 1]);
    };
    // a key's columns of P into the buffer
    auto store_p = [&](uint8_t* buf, const uint32_t (&x)[kH / 2]) {
        uint8_t* row = buf + (key >> 3) * F::kPGroup + (key & 7) * 128;
#pragma unroll
        for (int i = 0; i < kH / 8; ++i) {
            const int col = kC0 + 8 * i;
            *reinterpret_cast<uint4*>(row + (col >> 6) * 1024 + ((((col & 63) >> 3) ^ (key & 7)) << 4)) =
                make_uint4(x[4 * i], x[4 * i + 1], x[4 * i + 2], x[4 * i + 3]);
        }
    };

    look_up();
    load_row();
    Cursor cur = start;
    float l[kH];
    bool first_piece = true;
    uint32_t f_phase = 0;
    int piece_t0 = cur.t;
    decode(0);
    load_row();
    for (int j = 0; j < n_tiles; ++j) {
        const int L = s_len[cur.b], bg = p.b_base + cur.b;
        const int b2 = j & 1;
        const uint32_t ph = (uint32_t)(j >> 1) & 1;
        const bool first = j == 0 || cur.t == 0, last = j + 1 == n_tiles || cur.t + 1 == cur.T;
        if (first) {
            // ---- a new piece: its query rows as fp16 below 2^15 (as in the other form)
            piece_t0 = cur.t;
#pragma unroll
            for (int i = 0; i < kH; ++i) l[i] = 0.f;
            constexpr int kMine = (kN + 15) / 16;   // rows of a warp, requested together
            uint2 x[kMine];
            const float head = p.k_head ? __ldcg(p.k_head + cur.h) : 1.f;
#pragma unroll
            for (int k = 0; k < kMine; ++k) {
                const int row = warp + 16 * k;
                x[k] = make_uint2(0, 0);
                if (row < p.n_rows) {
                    const int i = s_draft[row];
                    const uint32_t* src = reinterpret_cast<const uint32_t*>(
                        p.q + (((size_t)bg * p.R + i) * p.Hq + (size_t)cur.h * p.G + (row - i * p.G)) * kPackDim + 4 * lane);
                    x[k].x = __ldcg(src);
                    x[k].y = __ldcg(src + 1);
                }
            }
#pragma unroll
            for (int k = 0; k < kMine; ++k) {
                const int row = warp + 16 * k;
                float back;
                const uint2 y = query_f16(x[k], back);
                if (row >= kN) continue;
                *reinterpret_cast<uint2*>(s_q + (lane >> 4) * F::kQHalf + row * 128 +
                                          ((((lane & 15) >> 1) ^ (row & 7)) << 4) + (lane & 1) * 8) = y;
                if (lane == 0) {
                    s_sc[row] = row < p.n_rows ? p.scale_log2 * back * head : 0.f;
                    s_up[row] = row < p.n_rows ? -kNegInf : 0.f;
                    s_m[row] = row < p.n_rows ? kNegInf : kPUp;
                }
            }
            fence_async_smem();
            workers_sync();
            k_arrive(j);
        }
        // ---- the next tile's row, once P and V of two tiles before are read
        if (j >= 2) tc_wait(&bars.o_done[b2], ph ^ 1, dead, p.status);
        if (j + 1 < n_tiles) {
            decode(j + 1);
            load_row();
            if (!last) k_arrive(j + 1);   // (a new piece's waits for its query rows)
        }
        // ---- softmax: this key's scores
        tc_wait(&bars.s_full[b2], ph, dead, p.status);
        tc_fence_after();
        float s[kH];
        const uint32_t s_at = tmem + lanes + F::kColS + b2 * kN + kC0;
#pragma unroll
        for (int i = 0; i < kH; i += 8) tc_ld8(s_at + i, s + i);
        tc_wait_ld();
        const int key0 = cur.t * kTcTile;
        const bool edge = key0 + kTcTile > L - p.R + 1;
        uint32_t pk[kH / 2], most = 0, least = 0x7c007c00u;
#pragma unroll
        for (int i = 0; i < kH; i += 4) {
            const float4 c = *reinterpret_cast<const float4*>(s_sc + kC0 + i), u = *reinterpret_cast<const float4*>(s_up + kC0 + i);
            float x0, x1, x2, x3;
            f2_unpack(f2_fma(f2_pack(s[i], s[i + 1]), f2_pack(c.x, c.y), f2_pack(u.x, u.y)), x0, x1);
            f2_unpack(f2_fma(f2_pack(s[i + 2], s[i + 3]), f2_pack(c.z, c.w), f2_pack(u.z, u.w)), x2, x3);
            s[i] = ex2(x0);
            s[i + 1] = ex2(x1);
            s[i + 2] = ex2(x2);
            s[i + 3] = ex2(x3);
            pk[i / 2] = pack_f16x2(s[i], s[i + 1]);
            pk[i / 2 + 1] = pack_f16x2(s[i + 2], s[i + 3]);
            most = max_f16x2(most, max_f16x2(pk[i / 2], pk[i / 2 + 1]));
            least = min_f16x2(least, min_f16x2(pk[i / 2], pk[i / 2 + 1]));
        }
        // (bits of positive fp16 numbers are in their order) above 2^15, below 2^-14
        const bool odd = max(most & 0xffffu, most >> 16) > 0x7800u || min(least & 0xffffu, least >> 16) < 0x0400u;
        int info = first ? 1 : 0;
        if (workers_any(odd || edge)) {
#pragma unroll
            for (int i = 0; i < kH; i += 8) tc_ld8(s_at + i, s + i);
            tc_wait_ld();
#pragma unroll
            for (int i = 0; i < kH; ++i) {
                const int row = kC0 + i;
                const int end = row < p.n_rows ? L - p.R + s_draft[row] : L - 1;
                s[i] = key0 + key <= end ? s[i] * s_sc[row] : kNegInf;
                const int top = __reduce_max_sync(0xffffffffu, ordered(s[i]));
                if (lane == 0) s_red[quad * kN + row] = top;
            }
            workers_sync();
            bool grew = false;
            if (key < kH) {
                const int row = kC0 + key;
                const float now = unordered(max(max(s_red[row], s_red[kN + row]), max(s_red[2 * kN + row], s_red[3 * kN + row])));
                const float m = s_m[row];
                float a = 1.f;
                if (row < p.n_rows && now - m > kPMax - kPUp) {   // (true for the first key: m is -inf)
                    a = ex2(m - now);
                    s_m[row] = now;
                    s_up[row] = kPUp - now;
                    grew = !first;
                }
                s_alpha[row] = a;
            }
            const bool rescale = workers_any(grew);
            auto is_faint = [&](float x) { return x < kPMin && x > kPGone; };
            bool faint = false;
#pragma unroll
            for (int i = 0; i < kH; ++i) {
                l[i] *= s_alpha[kC0 + i];
                s[i] = s[i] == kNegInf ? kNegInf : s[i] + s_up[kC0 + i];
                faint |= is_faint(s[i]);
            }
            faint = workers_any(faint);
            if ((rescale || faint) && j > 0) {
                tc_wait(&bars.o_done[b2 ^ 1], (uint32_t)((j - 1) >> 1) & 1, dead, p.status);
                tc_fence_after();
            }
            const uint32_t o_at = tmem + lanes + F::kColO + kC0;
            if (rescale) {
#pragma unroll 1
                for (int i = 0; i < kH; i += 8) {
                    float o[8];
                    uint32_t r[8];
                    tc_ld8(o_at + i, o);
                    tc_wait_ld();
#pragma unroll
                    for (int k = 0; k < 8; ++k) r[k] = __float_as_uint(o[k] * s_alpha[kC0 + i + k]);
                    tc_st8(o_at + i, r);
                }
                tc_wait_st();
            }
            for (float up = 28.f; faint; up += 28.f) {
                // this turn's weights through the tile's P, their product into its S (both free yet)
                uint32_t pf[kH / 2];
#pragma unroll
                for (int i = 0; i < kH; i += 2) {
                    float f[2];
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const float x = s[i + e];
                        const bool now = x < kPMin && x + up >= kPMin;
                        f[e] = now ? ex2(x + up) : 0.f;
                        if (now) {
                            l[i + e] += ex2(x);
                            s[i + e] = kNegInf;
                        }
                    }
                    pf[i / 2] = pack_f16x2(f[0], f[1]);
                }
                store_p(s_p + b2 * F::kPBytes, pf);
                fence_async_smem();
                tc_fence_before();
                workers_sync();
                tc_fence_after();
                if (warp == 0 && alive(dead) && elect_one()) {
                    tc_mma_values<kN>(tmem + F::kColS + b2 * kN, smem, j, false);
                    tc_commit(&bars.f_done);
                }
                __syncwarp();
                tc_wait(&bars.f_done, f_phase, dead, p.status);
                f_phase ^= 1;
                tc_fence_after();
                const float down = ex2(-up);
#pragma unroll 1
                for (int i = 0; i < kH; i += 8) {
                    float o[8], f[8];
                    uint32_t r[8];
                    tc_ld8(s_at + i, f);
                    tc_ld8(o_at + i, o);
                    tc_wait_ld();
                    // (a piece's first tile finds no sums yet)
#pragma unroll
                    for (int k = 0; k < 8; ++k) r[k] = __float_as_uint(info ? f[k] * down : fmaf(f[k], down, o[k]));
                    tc_st8(o_at + i, r);
                }
                tc_wait_st();
                info = 0;
                bool more = false;
#pragma unroll
                for (int i = 0; i < kH; ++i) more |= is_faint(s[i]);
                tc_fence_before();
                faint = workers_any(more);
            }
#pragma unroll
            for (int i = 0; i < kH; i += 2) {
                s[i] = ex2(s[i]);
                s[i + 1] = ex2(s[i + 1]);
                pk[i / 2] = pack_f16x2(s[i], s[i + 1]);
            }
        }
#pragma unroll
        for (int i = 0; i < kH; i += 2) f2_unpack(f2_add(f2_pack(l[i], l[i + 1]), f2_pack(s[i], s[i + 1])), l[i], l[i + 1]);
        store_p(s_p + b2 * F::kPBytes, pk);
        if (threadIdx.x == 0) s_info[b2] = info;
        fence_async_smem();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&bars.p_full[b2]);
        if (!last) {
            advance(cur, s_len, nb, p.Hkv, kTcTile);
            continue;
        }
        // ---- the end of a piece: sums over the keys, then a dim a thread
        const bool whole = piece_t0 == 0 && cur.t + 1 == cur.T;
        const int out_slot = 2 * cta + (first_piece ? 0 : 1);
        float* s_sum = reinterpret_cast<float*>(s_red);
#pragma unroll
        for (int i = 0; i < kH; ++i) {
#pragma unroll
            for (int off = 16; off > 0; off >>= 1) l[i] += __shfl_xor_sync(0xffffffffu, l[i], off);
            if (lane == 0) s_sum[quad * kN + kC0 + i] = l[i];
        }
        workers_sync();
        if (key < kH) {
            const int row = kC0 + key;
            const float sum = s_sum[row] + s_sum[kN + row] + s_sum[2 * kN + row] + s_sum[3 * kN + row];
            s_inv[row] = sum > 0.f ? (p.v_head ? __ldcg(p.v_head + cur.h) : 1.f) / sum : sum == 0.f ? 0.f : sum;
            if (!whole && row < p.n_rows) p.part_ml[(size_t)out_slot * p.n_rows + row] = make_float2(s_m[row], sum);
        }
        tc_wait(&bars.o_done[b2], ph, dead, p.status);
        tc_fence_after();
        workers_sync();   // (s_inv)
#pragma unroll 1
        for (int i = 0; i < kH; i += 8) {
            float o[8];
            tc_ld8(tmem + lanes + F::kColO + kC0 + i, o);
            tc_wait_ld();
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const int row = kC0 + i + k;
                if (row >= p.n_rows) continue;
                const float v = o[k] * s_inv[row];
                const int d = s_draft[row];
                if (whole)
                    p.out[(((size_t)bg * p.R + d) * p.Hq + (size_t)cur.h * p.G + (row - d * p.G)) * kPackDim + key] =
                        __float2bfloat16(v);
                else
                    p.part_o[((size_t)out_slot * p.n_rows + row) * kPackDim + key] = v;
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
        advance(cur, s_len, nb, p.Hkv, kTcTile);
        workers_sync();   // (the columns' words are free)
    }
}

template <int kN>
__global__ void __launch_bounds__(kTcThreads, 1) packed_attention_tc_kernel(const PackedAttnParams p) {
    using F = TcForm<kN>;
    extern __shared__ uint4 smem_raw[];
    uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    __shared__ TcBars bars;
    __shared__ long long s_wsum[kTcThreads / 32];
    __shared__ alignas(16) int s_info[8];      // [2] whether a tile's product starts O; then U and the CTAs
    __shared__ uint32_t s_tmem;
    __shared__ volatile int s_dead;
    __shared__ int s_draft[kN];
    int* s_len = reinterpret_cast<int*>(smem + F::kOffLen);
    long long* s_prefix = reinterpret_cast<long long*>(smem);
    const int warp = threadIdx.x >> 5, cta = blockIdx.x, grid = gridDim.x;
    const int nb = p.n_batch;
    if (threadIdx.x == 0) {
        s_dead = 0;
        for (int i = 0; i < 2; ++i) {
            mbar_init(&bars.k_full[i], 8);
            mbar_init(&bars.s_full[i], 1);
            mbar_init(&bars.p_full[i], 16);
            mbar_init(&bars.o_done[i], 1);
        }
        mbar_init(&bars.f_done, 1);
        fence_barrier_init();
    }
    for (int row = threadIdx.x; row < kN; row += kTcThreads) s_draft[row] = row / p.G;
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
        for (int b = threadIdx.x; b < nb; b += kTcThreads) s_prefix[b] += (long long)X * p.Hkv * b;
        __syncthreads();
    }
    const long long U = W + (long long)X * p.Hkv * nb;
    const Share share = share_of(cta, U, Gc, s_prefix, s_len, nb, p.Hkv, X, kTcTile);
    const int n_tiles = share.n_tiles;
    if (n_tiles <= 0) return;
    if (threadIdx.x == 0) {
        *reinterpret_cast<long long*>(s_info + 2) = U;
        s_info[4] = Gc;
    }
    if (warp == 16) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_u32(&s_tmem)) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();   // the prefix gives way to V
    tc_fence_after();
    const uint32_t tmem = s_tmem;

    const int group = warp >> 2;
    if (group < 2) {
        tc_worker<kN, F::kH0>(p, smem, bars, tmem, &s_dead, s_info, s_len, share.first, n_tiles, s_draft, group * F::kH0);
    } else if (group < 4) {
        tc_worker<kN, F::kH1>(p, smem, bars, tmem, &s_dead, s_info, s_len, share.first, n_tiles, s_draft,
                              2 * F::kH0 + (group - 2) * F::kH1);
    } else {
        // ---- the MMAs: S of tile j as soon as its K is there, O of tile j - 1
        // after it -- or before it where tile j opens a piece, whose query rows
        // wait for the end of the one before.  (Each wait names the phase that
        // follows the last one this warp has seen of its barrier.)
        const uint64_t dq = tc_desc(smem_u32(smem + F::kOffQ), 1024, 0);
        constexpr uint32_t id_s = tc_idesc(kN, false, false);
        uint64_t* open = nullptr;     // the latest commit
        uint32_t open_ph = 0;
        auto scores = [&](int j) {
            tc_wait(&bars.k_full[j & 1], (uint32_t)(j >> 1) & 1, &s_dead, p.status);
            tc_fence_after();
            __syncwarp();
            if (alive(&s_dead) && elect_one()) {
#pragma unroll
                for (int ks = 0; ks < kPackDim / 16; ++ks)
                    tc_mma_ts(tmem + F::kColS + (j & 1) * kN, tmem + (j & 1) * 64 + ks * 8,
                              dq + (uint64_t)((ks >> 2) * (F::kQHalf >> 4) + (ks & 3) * 2), id_s, ks > 0 ? 1u : 0u);
                tc_commit(&bars.s_full[j & 1]);
            }
            __syncwarp();
            open = &bars.s_full[j & 1];
            open_ph = (uint32_t)(j >> 1) & 1;
        };
        auto sums = [&](int j) {
            tc_wait(&bars.p_full[j & 1], (uint32_t)(j >> 1) & 1, &s_dead, p.status);
            tc_fence_after();
            const int info = *reinterpret_cast<volatile int*>(s_info + (j & 1));
            __syncwarp();
            if (alive(&s_dead) && elect_one()) {
                tc_mma_values<kN>(tmem + F::kColO, smem, j, !(info & 1));
                tc_commit(&bars.o_done[j & 1]);
            }
            __syncwarp();
            open = &bars.o_done[j & 1];
            open_ph = (uint32_t)(j >> 1) & 1;
        };
        Cursor cur = share.first;
        for (int j = 0; j < n_tiles; ++j) {
            if (j > 0) advance(cur, s_len, nb, p.Hkv, kTcTile);
            if (j > 0 && cur.t == 0) sums(j - 1);
            scores(j);
            if (j > 0 && cur.t != 0) sums(j - 1);
        }
        sums(n_tiles - 1);
        // every MMA completes before the tensor memory is given back
        if (!mbar_wait_bounded(open, open_ph) && (threadIdx.x & 31) == 0) atomicOr(p.status, CS_DEVICE_WAIT_TIMEOUT);
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (warp == 16) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem) : "memory");
}
