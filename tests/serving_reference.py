"""Plain references of the packed cache, the page operations and the log
probabilities, from their definitions: numpy, 64 bits (the quantisation in the
fp32 steps that define it)."""
import numpy as np

E2M1 = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def bf16(x):
    """fp64 -> the nearest bf16 value (ties to even), as fp64."""
    x = np.asarray(x, np.float32)
    b = x.view(np.uint32)
    r = ((b + 0x7FFF + ((b >> 16) & 1)) & 0xFFFF0000).astype(np.uint32)
    return np.where(np.isfinite(x), r.view(np.float32), x).astype(np.float64)


# ------------------------------------------------------------ packed format
def e4m3_values():
    """The value of every e4m3 byte (NaN for 0x7f and 0xff)."""
    b = np.arange(256)
    e, m = b >> 3 & 15, b & 7
    v = np.where(e == 0, m * 2.0 ** -9, (1 + m / 8) * 2.0 ** (e - 7.0))
    v = np.where((b & 0x7F) == 0x7F, np.nan, v)
    return np.where(b & 0x80, -v, v)


_POSITIVE = e4m3_values()[:0x7F]


def to_e4m3(x):
    """The byte of the e4m3 value nearest to 0 <= x <= 448, ties to the even byte."""
    x = np.asarray(x, np.float64)
    hi = np.clip(np.searchsorted(_POSITIVE, x), 1, len(_POSITIVE) - 1)
    lo = hi - 1
    dl, dh = x - _POSITIVE[lo], _POSITIVE[hi] - x
    return np.where((dh < dl) | ((dh == dl) & (hi % 2 == 0)), hi, lo).astype(np.uint8)


def quantise(x, head):
    """Codes uint8 [..., H, 64] and scale bytes [..., H, 8] of rows x (float array [..., H, 128])."""
    with np.errstate(all="ignore"):
        x = np.asarray(x, np.float32)
        head = np.asarray(head, np.float32)[:, None]
        g = np.where(np.isnan(x), np.float32(0), x).reshape(x.shape[:-1] + (8, 16))
        s = to_e4m3(np.minimum(np.abs(g).max(-1) / (np.float32(6) * head), np.float32(448)))
        unit = (_POSITIVE[s].astype(np.float32) * head)[..., None]
        q = np.where(unit > 0, g / unit, np.float32(0)).reshape(x.shape)
    a = np.minimum(np.abs(q).astype(np.float64), 6.0)
    hi = np.clip(np.searchsorted(E2M1, a), 1, 7)
    lo = hi - 1
    dl, dh = a - E2M1[lo], E2M1[hi] - a
    code = np.where((dh < dl) | ((dh == dl) & (hi % 2 == 0)), hi, lo) + 8 * np.signbit(q)
    code = code.astype(np.uint8)
    return code[..., 0::2] | (code[..., 1::2] << 4), s


def values(codes, scales, head):
    """fp64 rows [..., H, n, 128] of codes [..., H, n, 64] and scale bytes [..., H, n, 8]."""
    c = np.stack((codes & 15, codes >> 4), -1).reshape(codes.shape[:-1] + (128,))
    v = E2M1[c & 7] * np.where(c & 8, -1.0, 1.0)
    s = e4m3_values()[scales].repeat(16, axis=-1)
    return v * s * np.asarray(head, np.float64)[:, None, None]


def place(table, lens, n, ps, P):
    """(b, i, page, slot) of every row that an append of n rows writes."""
    cap = table.shape[1] * ps
    for b, L in enumerate(lens):
        L = min(max(int(L), 0), cap)
        for i in range(n):
            pos = L - n + i
            if pos >= 0 and 0 <= table[b, pos // ps] < P:
                yield b, i, int(table[b, pos // ps]), pos % ps


def packed_attention(q, k, v, table, lens, scale):
    """out [B, R, Hq, D] and sum_j p_j |v_j|, from fp64 pools k, v [P, Hkv, ps, D]."""
    B, R, Hq, D = q.shape
    P, Hkv, ps, _ = k.shape
    out, size = np.zeros(q.shape), np.zeros(q.shape)
    for b in range(B):
        L = min(max(int(lens[b]), 0), table.shape[1] * ps)
        if L == 0:
            continue
        kk, vv = np.zeros((Hkv, L, D)), np.zeros((Hkv, L, D))
        for j0 in range(0, L, ps):
            page, n = table[b, j0 // ps], min(ps, L - j0)
            if 0 <= page < P:
                kk[:, j0:j0 + n], vv[:, j0:j0 + n] = k[page, :, :n], v[page, :, :n]
        for i in range(R):
            n = L - R + 1 + i
            if n <= 0:
                continue
            x = q[b, i].reshape(Hkv, Hq // Hkv, D)
            s = np.einsum("hgd,hld->hgl", x, kk[:, :n]) * scale
            p = np.exp(s - s.max(-1, keepdims=True))
            p /= p.sum(-1, keepdims=True)
            out[b, i] = np.einsum("hgl,hld->hgd", p, vv[:, :n]).reshape(Hq, D)
            size[b, i] = np.einsum("hgl,hld->hgd", p, np.abs(vv[:, :n])).reshape(Hq, D)
    return out, size


# -------------------------------------------------------------------- pages
def fork(pools, table, lens, refs, src, dst, ps, room):
    """In place; returns what was forked."""
    R, cols = table.shape
    P = len(refs)
    free = [p for p in range(P) if refs[p] == 0]
    taken, done = 0, []
    for s, d in zip(src, dst):
        valid = -1 <= s < R and 0 <= d < R
        L = min(max(int(lens[s]), 0), cols * ps) if valid and s >= 0 else 0
        full = L // ps
        own = -(-min(L + room, cols * ps) // ps) - full if valid else 0
        ok = valid and taken + own <= len(free)
        mine = free[taken:taken + own] if ok else []
        taken += own
        done.append(int(ok))
        if not 0 <= d < R:
            continue
        row = np.full(cols, -1, np.int32)
        if ok:
            row[:full] = table[s, :full] if full else row[:full]
            for p in row[:full]:
                if 0 <= p < P:
                    refs[p] += 1
            row[full:full + own] = mine
            for p in mine:
                refs[p] = 1
            if L % ps and 0 <= table[s, full] < P:
                for pool in pools:
                    pool[mine[0]] = pool[table[s, full]]
        table[d] = row
        lens[d] = L if ok else 0
    return np.array(done, np.int32)


def release(table, lens, refs, rows, keep, ps):
    R, cols = table.shape
    for r, k in zip(rows, keep):
        if not 0 <= r < R:
            continue
        k = min(max(int(k), 0), cols * ps)
        for j in range(-(-k // ps), cols):
            if 0 <= table[r, j] < len(refs):
                refs[table[r, j]] -= 1
            table[r, j] = -1
        lens[r] = min(lens[r], k)


def compact(pools, table, refs):
    live = [p for p in range(len(refs)) if refs[p] != 0]
    N = len(live)
    of = [p for p in live if p >= N]
    to = [p for p in range(N) if refs[p] == 0]
    where = dict(zip(of, to))
    for a, b in where.items():
        for pool in pools:
            pool[b] = pool[a]
        refs[b], refs[a] = refs[a], 0
    for e in np.ndindex(table.shape):
        table[e] = where.get(int(table[e]), table[e])
    return N


# -------------------------------------------------------- log probabilities
def logprobs(z, tokens, T, n_top):
    """z fp64 [N, V]: (lp, entropy, top ids, top lp)."""
    N, V = z.shape
    lp, ent = np.full(N, -np.inf), np.zeros(N)
    ids, top = np.full((N, n_top), -1, np.int32), np.full((N, n_top), -np.inf)
    for r in range(N):
        m = z[r].max()
        if tokens[r] < 0 or m == -np.inf:
            continue
        d = (z[r] - m) / T
        lse = np.log(np.exp(d).sum())
        p = np.exp(d - lse)
        if tokens[r] < V:
            lp[r] = d[tokens[r]] - lse
        on = p > 0
        ent[r] = -(p[on] * (d[on] - lse)).sum()
        order = np.argsort(-z[r], kind="stable")[:n_top]
        order = order[z[r][order] > -np.inf]
        ids[r, :len(order)] = order
        top[r, :len(order)] = d[order] - lse
    return lp, ent, ids, top
