// ragged.cuh -- the rows of a batch whose requests have different numbers of new
// tokens (cs_rope_kv_append, cs_chunk_attention): which request a token belongs to.
#pragma once

#include "cs_device.cuh"

namespace cs {

// Quotients by a divisor that the host knows, of numbers below 2^31: one high product
// and a shift (Granlund and Montgomery, 1994).
struct HostDivisor {
    uint32_t d, mul;
    int shift;
    static HostDivisor of(uint32_t d) {
        HostDivisor x{d, 0, 0};
        while ((1ull << x.shift) < d) ++x.shift;
        if (x.shift > 0) x.mul = (uint32_t)(((1ull << (31 + x.shift)) + d - 1) / d);
        return x;
    }
    __device__ __forceinline__ uint32_t operator()(uint32_t n) const {
        return shift > 0 ? __umulhi(n, mul) >> (shift - 1) : n;
    }
};

struct RaggedBatch {
    const int32_t* ctx_lens;   // [B]
    const int32_t* q_starts;   // [B + 1], or NULL: n rows each
    int B, tokens, n;
    int max_keys;              // keys that a row of the page table can hold

    // Request b's rows, [start, start + n), in [0, tokens], and its length
    __device__ __forceinline__ void rows_of(int b, int& start, int& count, int& len) const {
        len = max(0, min(__ldcg(ctx_lens + b), max_keys));
        if (!q_starts) {
            start = b * n;
            count = n;
            return;
        }
        start = max(0, min(__ldcg(q_starts + b), tokens));
        count = max(0, min(__ldcg(q_starts + b + 1), tokens) - start);
    }

    // The request that token t may belong to (the whole warp asks for one token), the last
    // one that does not begin behind it; -1: none.  Whether it does, its rows say.  32 places
    // of the array at a time: two loads up to 1024 requests.
    __device__ __forceinline__ int request_of(int t, int lane) const {
        if (!q_starts) return t / n < B ? t / n : -1;
        int lo = 0, len = B + 1;   // the last b with q_starts[b] <= t lies in [lo, lo + len), if anywhere
        while (len > 1) {
            const int step = (len + 31) / 32;
            const int at = lo + lane * step;
            const unsigned before = __ballot_sync(0xffffffffu, lane * step < len && __ldcg(q_starts + at) <= t);
            if (before == 0) return -1;
            const int last = 31 - __clz(before);
            lo += last * step;
            len = min(step, len - last * step);
        }
        return lo < B ? lo : -1;
    }
};

}  // namespace cs
