"""Plain references of the operators over requests with different numbers of new
tokens, from their definitions, in 64 bits (torch)."""
import math

import torch


def rows_of(starts, lens, B, T, cap):
    """(request, row, its place among the request's, its key position) of every token that belongs to a request."""
    for b in range(B):
        s, e = (b * T // B, (b + 1) * T // B) if starts is None else (int(starts[b]), int(starts[b + 1]))
        L = min(max(int(lens[b]), 0), cap)
        for i in range(e - s):
            yield b, s + i, i, L - (e - s) + i


def turn(x, t, cos_sin, norm, eps, interleaved):
    """64-bit heads x [H, 128] of a token at rotation position t."""
    x = x.double().clone()
    if norm is not None:
        x = x * norm.double() / torch.sqrt(x.square().mean(-1, keepdim=True) + eps)
    half = cos_sin.shape[1] // 2
    c, s = cos_sin[t, :half].double(), cos_sin[t, half:].double()
    out = x.clone()
    for i in range(half):
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
        out[:, a] = x[:, a] * c[i] - x[:, b] * s[i]
        out[:, b] = x[:, b] * c[i] + x[:, a] * s[i]
    return out


def attention(q, k_pages, v_pages, table, lens, starts, scale=None):
    """(out, sum_j p_j |v_j|) [T, Hq, 128] in 64 bits, zeros in rows of nobody; on the tensors' device."""
    T, Hq, D = q.shape
    P, Hkv, ps, _ = k_pages.shape
    G, B, cap = Hq // Hkv, table.shape[0], table.shape[1] * ps
    scale = 1 / math.sqrt(D) if scale is None else scale
    out, size = (torch.zeros(q.shape, dtype=torch.float64, device=q.device) for _ in range(2))
    where, length = table.tolist(), lens.tolist()
    first = None if starts is None else starts.tolist()
    for b in range(B):
        s, e = (b * T // B, (b + 1) * T // B) if first is None else (first[b], first[b + 1])
        n, L = e - s, min(max(length[b], 0), cap)
        if n == 0 or L == 0:
            continue
        ids = torch.tensor(where[b][:-(-L // ps)], device=q.device)
        there = ((ids >= 0) & (ids < P))[:, None, None, None]
        k, v = (torch.where(there, p[ids.clamp(0, P - 1)], 0).transpose(0, 1).flatten(1, 2)[:, :L].double()
                for p in (k_pages, v_pages))
        x = q[s:e].double().unflatten(1, (Hkv, G))
        t = torch.einsum("nhgd,hld->hgnl", x, k) * scale
        seen = torch.arange(L, device=q.device)[None] <= (L - n + torch.arange(n, device=q.device))[:, None]
        p = torch.softmax(t.masked_fill(~seen, -math.inf), -1)
        p = torch.where(seen.any(1)[:, None], p, torch.zeros_like(p))
        out[s:e] = torch.einsum("hgnl,hld->nhgd", p, v).flatten(1, 2)
        size[s:e] = torch.einsum("hgnl,hld->nhgd", p, v.abs()).flatten(1, 2)
    return out, size
