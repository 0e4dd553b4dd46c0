"""The operators that take a prompt's tokens through the paged cache, as cases that can be timed and compared.

* ``chunk``: attention of every request's newest tokens over the paged bf16
  cache, causal among them; a request has a number of them of its own, from one
  to a whole chunk of its prompt;
* ``rope``: rotating the queries and keys of new tokens by their positions
  (after a norm of each head, where a model has one) and appending keys and
  values to the bf16 cache;
* ``packed``: the same into the cache held in 4 bits (e2m1 codes, an e4m3 scale
  for 16 dims, an fp32 scale for each KV head), and the rows read back.

Where ``own`` is false a pass computes the operators in their plain form.
"""
from __future__ import annotations

import math

import torch

own = False   # whether run() makes the library's calls or computes the plain form

DEVICE = "cuda:0"
D = 128          # head dim
GROUP = 16       # dims that share a scale
EPS = 1e-6
E2M1 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
_HEADS = ((32, 8), (28, 4), (64, 8), (16, 4), (32, 32), (40, 8))


# --------------------------------------------------------------------------
# the cases
# --------------------------------------------------------------------------
def _chunk(batch, single, nlo, nhi, plo, phi, hq, hkv, page, fused):
    """The first ``single`` of ``batch`` requests have one new token, the others nlo .. nhi; plo .. phi before them.
    fused: the queries lie in the rows of a projection of queries, keys and values."""
    return dict(op="chunk", batch=batch, single=single, nlo=nlo, nhi=nhi, plo=plo, phi=phi, hq=hq, hkv=hkv, page=page,
                fused=fused)


def _rope(op, batch, nlo, nhi, plo, phi, hq, hkv, page, rot, pairs, norm, tree):
    """rot: dims that turn; pairs: "halves" (i, i + rot/2) or "neighbours" (2i, 2i + 1); tree: the new tokens are a
    tree's nodes, whose positions are given."""
    return dict(op=op, batch=batch, single=0, nlo=nlo, nhi=nhi, plo=plo, phi=phi, hq=hq, hkv=hkv, page=page, rot=rot,
                pairs=pairs, norm=norm, tree=tree)


def listed():
    return [
        # one interactive request, a token at a time: latency
        dict(name="chunk-b1-single", **_chunk(1, 1, 1, 1, 511, 511, 32, 8, 16, False)),
        # a short prompt at once, nothing before it
        dict(name="chunk-b1-prompt", **_chunk(1, 0, 777, 777, 0, 0, 32, 8, 16, True)),
        # a full server without drafts: the cache's bytes and little else
        dict(name="chunk-b128-single", **_chunk(128, 128, 1, 1, 1023, 8191, 64, 8, 32, False)),
        # continuous batching: chunks of prompts beside requests that decode, seven query heads a KV head
        dict(name="chunk-b24-mixed", **_chunk(24, 20, 301, 512, 63, 4095, 28, 4, 16, True)),
        # the prompts of a burst of requests of a model whose query heads share no keys
        dict(name="chunk-b8-prompts", **_chunk(8, 0, 129, 1024, 0, 1024, 32, 32, 64, True)),
        # a chunk of a long document: the largest call
        dict(name="chunk-b1-long", **_chunk(1, 0, 4096, 4096, 12288, 12288, 64, 8, 16, False)),
        # one interactive request's token: latency
        dict(name="rope-b1-single", **_rope("rope", 1, 1, 1, 100, 511, 32, 8, 16, 128, "halves", False, False)),
        # the rows of a verify step of drafted trees, the heads normed
        dict(name="rope-b64-tree", **_rope("rope", 64, 21, 21, 64, 512, 28, 4, 16, 128, "halves", True, True)),
        # the chunks of a burst of prompts
        dict(name="rope-b16-prompts", **_rope("rope", 16, 1500, 2049, 0, 64, 64, 8, 16, 128, "halves", True, False)),
        # a model that turns half of each head, by neighbouring pairs
        dict(name="rope-b5-partial", **_rope("rope", 5, 33, 700, 0, 300, 40, 8, 32, 64, "neighbours", False, False)),
        # a token for each request of a full server
        dict(name="packed-b256-single", **_rope("packed", 256, 1, 1, 64, 512, 32, 8, 16, 128, "halves", True, False)),
        # prompts into the packed cache
        dict(name="packed-b8-prompts", **_rope("packed", 8, 2049, 2049, 0, 500, 32, 8, 16, 128, "halves", False, False)),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(("chunk", "chunk", "chunk", "rope", "rope", "packed"))
    page = rng.choice((16, 16, 32, 64))
    hq, hkv = rng.choice(_HEADS)
    while op == "chunk":
        batch, nhi, phi = _log_int(rng, 1, 128), _log_int(rng, 1, 4096), _log_int(rng, 1, 12288) - 1
        nlo, plo = _log_int(rng, 1, nhi), _log_int(rng, 1, phi + 1) - 1
        single = rng.choice((0, 0, batch // 2, batch))
        if single == batch:
            nlo = nhi = 1
        # at most the scores of the plain form and the keys of the largest listed cases
        if (batch * nhi * hq * (phi + nhi) <= 64 * 4096 * 16384 and batch * hkv * (phi + nhi) <= 128 * 8 * 8192):
            return _chunk(batch, single, nlo, nhi, plo, phi, hq, hkv, page, rng.random() < 0.5)
    while True:
        batch, nhi, phi = _log_int(rng, 1, 256), _log_int(rng, 1, 4096), _log_int(rng, 1, 4096) - 1
        nlo, plo = (nhi if op == "packed" else _log_int(rng, 1, nhi)), _log_int(rng, 1, phi + 1) - 1
        tree = nhi <= 64 and rng.random() < 0.3
        if batch * nhi * (hq + 2 * hkv) <= 16 * 2049 * 80 and batch * (phi + nhi) * hkv <= 1 << 23:
            return _rope(op, batch, nlo, nhi, plo, phi, hq, hkv, page, rng.choice((128, 128, 64, 32)),
                         rng.choice(("halves", "halves", "neighbours")), rng.random() < 0.5, tree)


# --------------------------------------------------------------------------
# the packed format
# --------------------------------------------------------------------------
def _quantise(x, head):
    """Codes (two dims a byte, the even one low) and e4m3 scales of fp32 rows x [..., H, D]; head: fp32 [H]."""
    g = x.unflatten(-1, (D // GROUP, GROUP))
    s = (g.abs().amax(-1) / (6.0 * head[:, None])).clamp(max=448.0).to(torch.float8_e4m3fn)
    unit = (s.float() * head[:, None])[..., None]
    q = torch.where(unit > 0, g / unit, torch.zeros_like(g))
    a = q.abs()
    # nearest, ties to the even code
    code = ((a > 0.25).byte() + (a >= 0.75) + (a > 1.25) + (a >= 1.75) + (a > 2.5) + (a >= 3.5) + (a > 5.0)
            + 8 * torch.signbit(q)).byte().flatten(-2)
    return code[..., 0::2] | (code[..., 1::2] << 4), s


def _dequantise(codes, scales, head):
    """fp32 rows [..., H, D] of codes [..., H, D / 2] and scales [..., H, D / 16]."""
    one = torch.tensor(E2M1 + tuple(-v for v in E2M1), dtype=torch.float32, device=codes.device)
    byte = torch.arange(256, device=codes.device)
    both = torch.stack((one[byte & 15], one[byte >> 4]), dim=1)
    x = both[codes.int()].flatten(-2).unflatten(-1, (D // GROUP, GROUP))
    return (x * (scales.float() * head[:, None])[..., None]).flatten(-2)


# --------------------------------------------------------------------------
# inputs
# --------------------------------------------------------------------------
def _counts(case):
    """The numbers of new tokens and of tokens before them of a case's requests, spread evenly over their ranges (in
    orders of their own; the largest of both are one request's)."""
    B, many = case["batch"], case["batch"] - case["single"]
    spread = lambda lo, hi, m, step: [lo + (hi - lo) * (i * step % m) // max(m - 1, 1) for i in range(1, m)] + [hi]  # noqa: E731
    n = [1] * case["single"] + (spread(case["nlo"], case["nhi"], many, 1) if many else [])
    step = next(k for k in range(int(0.618 * B) + 1, 2 * B + 2) if math.gcd(k, B) == 1)
    return n, spread(case["plo"], case["phi"], B, step)


def _tables(lens, max_pages, page, pages, gen):
    """A page table of rows whose pages lie anywhere in the pool, -1 past each row's last."""
    order = torch.randperm(pages, generator=gen, device=DEVICE).int()
    need = (lens + page - 1) // page
    col = torch.arange(max_pages, device=DEVICE)[None]
    at = (torch.cumsum(need, 0) - need)[:, None] + col
    held = col < need[:, None]
    return torch.where(held, order[at.clamp(max=pages - 1)], torch.full_like(held, -1, dtype=torch.int32)).contiguous()


def prepare(case, seed):
    gen = torch.Generator(device=DEVICE).manual_seed(seed)
    B, hq, hkv, page = case["batch"], case["hq"], case["hkv"], case["page"]
    order = torch.randperm(B, generator=torch.Generator().manual_seed(seed))
    n, before = (torch.tensor(c)[order] for c in _counts(case))
    T, longest = int(n.sum()), int((n + before).max())
    max_pages = -(-longest // page)
    starts = torch.zeros(B + 1, dtype=torch.int32)
    starts[1:] = torch.cumsum(n, 0)
    s = dict(case=case, tokens=T, widest=int(n.max()), starts=starts.to(DEVICE), lens=(n + before).int().to(DEVICE))
    pages = int(((n + before + page - 1) // page).sum()) + 3
    s["table"] = _tables(s["lens"], max_pages, page, pages, gen)
    shape = (pages, hkv, page)
    normal = lambda *size: torch.empty(size, dtype=torch.bfloat16, device=DEVICE).normal_(generator=gen)  # noqa: E731
    if case["op"] == "packed":
        s["head"] = [2.0 ** (torch.rand(hkv, generator=gen, device=DEVICE) * 2 - 4) for _ in range(2)]
        s["pool"] = [torch.zeros(shape + (w,), dtype=t, device=DEVICE)
                     for _ in range(2) for w, t in ((D // 2, torch.uint8), (D // GROUP, torch.float8_e4m3fn))]
    else:
        s["pool"] = [normal(*shape, D) for _ in range(2)]
    if case["op"] == "chunk":
        s["q"] = normal(T, hq + 2 * hkv if case["fused"] else hq, D)[:, :hq]
        return s
    # the projection's rows: queries, keys, values
    rows = normal(T, hq + 2 * hkv, D)
    s["qkv"] = rows[:, :hq], rows[:, hq:hq + hkv], rows[:, hq + hkv:]
    rot = case["rot"]
    angle = (torch.arange(max_pages * page, device=DEVICE, dtype=torch.float64)[:, None]
             * 500000.0 ** (-torch.arange(0, rot, 2, device=DEVICE, dtype=torch.float64) / rot)[None])
    s["turns"] = torch.cat((angle.cos(), angle.sin()), 1).float().contiguous()
    s["norms"] = [(1 + 0.2 * torch.randn(D, generator=gen, device=DEVICE)).bfloat16() if case["norm"] else None
                  for _ in range(2)]
    s["positions"] = None
    if case["tree"]:   # the nodes' depths below the root, which is the first new token
        i = torch.arange(T, device=DEVICE) - s["starts"][:-1].repeat_interleave(n.to(DEVICE), output_size=T)
        root = before.to(DEVICE).repeat_interleave(n.to(DEVICE), output_size=T)
        s["positions"] = (root + torch.log2(i + 1.0).floor().long()).int()
    return s


# --------------------------------------------------------------------------
# one pass
# --------------------------------------------------------------------------
def run(state):
    return (_run_own if own else _run_plain)[state["case"]["op"]](state)


def _own_chunk(s):
    from paper_2607_20507_gb300 import binding
    return dict(out=binding.cs_chunk_attention(s["q"], *s["pool"], s["table"], s["lens"], s["starts"]))


def _own_rope(s):
    from paper_2607_20507_gb300 import binding
    q = binding.cs_rope_kv_append(*s["qkv"], s["turns"], *s["pool"], s["table"], s["lens"], s["starts"],
                                  positions=s["positions"], q_norm=s["norms"][0], k_norm=s["norms"][1], norm_eps=EPS,
                                  interleaved=s["case"]["pairs"] == "neighbours")
    return dict(q=q, k_pages=s["pool"][0], v_pages=s["pool"][1])


def _own_packed(s):
    from paper_2607_20507_gb300 import binding
    pool = binding.PackedPool(*s["pool"], *s["head"])
    q = binding.cs_packed_rope_kv_append(*s["qkv"], s["turns"], pool, s["table"], s["lens"], s["starts"],
                                         positions=s["positions"], q_norm=s["norms"][0], k_norm=s["norms"][1],
                                         norm_eps=EPS, interleaved=s["case"]["pairs"] == "neighbours")
    k, v = binding.cs_packed_kv_read(pool, s["table"], s["lens"], s["case"]["nhi"])
    return dict(q=q, k=k, v=v, k_scales=pool.k_scales, v_scales=pool.v_scales)


_run_own = dict(chunk=_own_chunk, rope=_own_rope, packed=_own_packed)


def _of_tokens(s):
    """Each token's request, its place among the request's new ones, and its key position."""
    n = (s["starts"][1:] - s["starts"][:-1]).long()
    b = torch.arange(n.shape[0], device=n.device).repeat_interleave(n, output_size=s["tokens"])
    i = torch.arange(s["tokens"], device=n.device) - s["starts"][:-1].long()[b]
    return b, i, s["lens"].long()[b] - n[b] + i


def _plain_chunk(s):
    q, (k_pages, v_pages), lens, starts = s["q"], s["pool"], s["lens"], s["starts"].long()
    hq, hkv, N = q.shape[1], k_pages.shape[1], s["widest"]
    dense = lambda pool: pool[s["table"].clamp(min=0)].transpose(1, 2).flatten(2, 3).float()   # noqa: E731  [B, H, L, D]
    at = (starts[:-1, None] + torch.arange(N, device=q.device)[None]).clamp(max=s["tokens"] - 1)
    x = q[at].float().unflatten(2, (hkv, hq // hkv)).permute(0, 2, 3, 1, 4).flatten(2, 3)     # [B, H, G N, D]
    score = (x @ dense(k_pages).transpose(2, 3)).mul_(1 / math.sqrt(D))
    last = (lens - (starts[1:] - starts[:-1]))[:, None] + torch.arange(N, device=q.device)[None]   # row i's last key
    hidden = torch.arange(score.shape[3], device=q.device)[None, None] > last[:, :, None]
    score.unflatten(2, (-1, N)).masked_fill_(hidden[:, None, None], -math.inf)
    p = torch.exp_(score.sub_(score.amax(-1, keepdim=True)))
    o = (p @ dense(v_pages)) / p.sum(-1, keepdim=True)
    o = o.unflatten(2, (-1, N)).permute(0, 3, 1, 2, 4).flatten(2, 3)     # [B, N, Hq, D]
    b, i, _ = _of_tokens(s)
    return dict(out=o[b, i].bfloat16())


def _plain_turn(s, x, norm, where):
    """fp32 heads x [T, H, D], normed and turned."""
    rot, x = s["case"]["rot"], x.float()
    if norm is not None:
        x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * norm.float()
    cos, sin = s["turns"][where][:, None].chunk(2, -1)
    if s["case"]["pairs"] == "neighbours":
        a, c = x[..., 0:rot:2], x[..., 1:rot:2]
        turned = torch.stack((a * cos - c * sin, c * cos + a * sin), -1).flatten(-2)
    else:
        a, c = x[..., :rot // 2], x[..., rot // 2:rot]
        turned = torch.cat((a * cos - c * sin, c * cos + a * sin), -1)
    return torch.cat((turned, x[..., rot:]), -1)


def _plain_rows(s):
    """The queries and keys, turned, the values, and their pages and slots."""
    b, _, j = _of_tokens(s)
    where = j if s["positions"] is None else s["positions"].long()
    q, k, v = s["qkv"]
    return (_plain_turn(s, q, s["norms"][0], where).bfloat16(), _plain_turn(s, k, s["norms"][1], where), v,
            s["table"][b, j // s["case"]["page"]].long(), j % s["case"]["page"])


def _plain_rope(s):
    q, k, v, page, slot = _plain_rows(s)
    k_pages, v_pages = s["pool"]
    k_pages[page, :, slot] = k.bfloat16()
    v_pages[page, :, slot] = v
    return dict(q=q, k_pages=k_pages, v_pages=v_pages)


def _plain_packed(s):
    q, k, v, page, slot = _plain_rows(s)
    kc, ks, vc, vs = s["pool"]
    out = []
    for x, c, z, h in ((k, kc, ks, s["head"][0]), (v.float(), vc, vs, s["head"][1])):
        code, scale = _quantise(x, h)
        c[page, :, slot] = code
        z[page, :, slot] = scale
        out.append(_dequantise(c[page, :, slot], z[page, :, slot], h).bfloat16().unflatten(0, (s["case"]["batch"], -1)))
    return dict(q=q, k=out[0], v=out[1], k_scales=ks, v_scales=vs)


_run_plain = dict(chunk=_plain_chunk, rope=_plain_rope, packed=_plain_packed)


# --------------------------------------------------------------------------
# what a pass cannot do without
# --------------------------------------------------------------------------
def work(case):
    B, hq, hkv = case["batch"], case["hq"], case["hkv"]
    n, before = _counts(case)
    T = sum(n)
    if case["op"] == "chunk":
        keys = T + sum(before)
        seen = sum(a * (2 * p + a + 1) / 2 for a, p in zip(n, before))   # (row, key) pairs of a head
        return dict(bytes=keys * (4 * hkv * D + 4 / case["page"]) + 4 * T * hq * D + 8 * B, flops=4 * D * hq * seen)
    row = D // 2 + D // GROUP        # one packed row of one head
    out = 2 * hkv * (2 * row + 2 * D) if case["op"] == "packed" else 4 * hkv * D   # packed: written, read, as bf16
    return dict(bytes=T * (2 * (2 * hq + 2 * hkv) * D + out + 4 * case["rot"]), flops=T * (hq + hkv) * (3 * case["rot"]))


# --------------------------------------------------------------------------
# the results from the definitions in 64 bits
# --------------------------------------------------------------------------
def _exact_chunk(case, s):
    q, starts, lens = s["q"], s["starts"].tolist(), s["lens"].tolist()
    out = torch.empty(q.shape, dtype=torch.float64, device=DEVICE)
    G = case["hq"] // case["hkv"]
    for b, L in enumerate(lens):
        rows = slice(starts[b], starts[b + 1])
        n = starts[b + 1] - starts[b]
        pages = s["table"][b, :-(-L // case["page"])].long()
        visible = torch.ones((n, L), dtype=torch.bool, device=DEVICE).tril(L - n)
        for h in range(case["hkv"]):
            k, v = (pool[pages, h].flatten(0, 1)[:L].double() for pool in s["pool"])
            for g in range(h * G, h * G + G):
                t = (q[rows, g].double() @ k.T / math.sqrt(D)).masked_fill_(~visible, -math.inf)
                out[rows, g] = torch.softmax(t, -1) @ v
    return dict(out=out)


def _exact_turn(case, s, x, norm):
    """64-bit heads x [T, H, D], normed, then turned as complex numbers."""
    x = x.double()
    if norm is not None:
        x = x / torch.sqrt(x.square().sum(-1, keepdim=True) / D + EPS) * norm.double()
    where = torch.cat([torch.arange(L - n, L, device=DEVICE) for L, n in
                       zip(s["lens"].tolist(), (s["starts"][1:] - s["starts"][:-1]).tolist())])
    where = where if s["positions"] is None else s["positions"].long()
    rot = case["rot"]
    turn = torch.complex(*s["turns"].double()[where][:, None].chunk(2, -1))
    head = x[..., :rot]
    if case["pairs"] == "neighbours":
        z = torch.view_as_complex(head.unflatten(-1, (-1, 2)).contiguous()) * turn
        head = torch.view_as_real(z).flatten(-2)
    else:
        z = torch.complex(*head.chunk(2, -1)) * turn
        head = torch.cat((z.real, z.imag), -1)
    return torch.cat((head, x[..., rot:]), -1)


def _exact_rope(case, s):
    q = _exact_turn(case, s, s["qkv"][0], s["norms"][0])
    k = _exact_turn(case, s, s["qkv"][1], s["norms"][1])
    pages = [p.double() for p in s["pool"]]
    starts, lens, table = s["starts"].tolist(), s["lens"].tolist(), s["table"].long()
    for b, L in enumerate(lens):
        n = starts[b + 1] - starts[b]
        at = torch.arange(L - n, L, device=DEVICE)
        page, slot = table[b, at // case["page"]], at % case["page"]
        pages[0][page, :, slot] = k[starts[b]:starts[b + 1]]
        pages[1][page, :, slot] = s["qkv"][2][starts[b]:starts[b + 1]].double()
    return dict(q=q, k_pages=pages[0], v_pages=pages[1])


def _exact_grid(x, head):
    """The values that 64-bit rows x [T, H, D] are held as."""
    h = head.double()[:, None, None]
    g = x.unflatten(-1, (D // GROUP, GROUP))
    s = g.abs().amax(-1, keepdim=True) / (6 * h)
    step = torch.exp2(torch.floor(torch.log2(s.clamp(min=2.0 ** -6))) - 3)      # of e4m3
    unit = (torch.round(s / step) * step).clamp(max=448.0) * h
    y = g / torch.where(unit > 0, unit, torch.ones_like(unit))
    a = y.abs().clamp(max=6.0)
    step = torch.where(a < 2, 0.5, torch.where(a < 4, 1.0, 2.0))               # of e2m1
    return (torch.round(a / step) * step * torch.sign(y) * unit).flatten(-2)


def _exact_packed(case, s):
    rows = lambda x, h: _exact_grid(x, h).unflatten(0, (case["batch"], -1))   # noqa: E731
    return dict(q=_exact_turn(case, s, s["qkv"][0], s["norms"][0]),
                k=rows(_exact_turn(case, s, s["qkv"][1], s["norms"][1]), s["head"][0]),
                v=rows(s["qkv"][2].double(), s["head"][1]), k_scales=None, v_scales=None)


def exact(case, seed):
    return dict(chunk=_exact_chunk, rope=_exact_rope, packed=_exact_packed)[case["op"]](case, prepare(case, seed))
