"""The operators around a packed K/V cache and a server's answers, as cases that can be timed and compared.

* ``attn``: verify attention over a cache held in 4 bits (e2m1 codes, an e4m3
  scale for 16 dims, an fp32 scale for each KV head), from single-token
  decoding to the k+1 positions of a draft;
* ``append``: quantising new K/V rows into that cache, and reading them back;
* ``logprobs``: log probabilities of given tokens with the entropy and the top
  alternatives of their rows;
* ``fork``: the samples of the last round give their pages back, the next ones
  share their prompt's;
* ``compact``: finished requests give their pages back, the pages in use move
  together.

Where ``own`` is false a pass computes the operators in their plain form.
"""
from __future__ import annotations

import math

import torch

own = False   # whether run() makes the library's calls or computes the plain form

DEVICE = "cuda:0"
D = 128          # head dim
GROUP = 16       # dims that share a scale
E2M1 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
_HEADS = ((32, 8), (28, 4), (64, 8), (16, 4), (32, 32), (40, 8))
_VOCABS = (32000, 128256, 151936, 256000)


# --------------------------------------------------------------------------
# the cases
# --------------------------------------------------------------------------
def _attn(batch, rows, hq, hkv, page, ctx, lo, hi):
    return dict(op="attn", batch=batch, rows=rows, hq=hq, hkv=hkv, page=page, ctx=ctx, lo=lo, hi=hi)


def _append(batch, n_new, hkv, page, lo, hi):
    return dict(op="append", batch=batch, n_new=n_new, hkv=hkv, page=page, lo=lo, hi=hi)


def _logprobs(batch, rows, vocab, dtype, top, temperature, masked, emitted):
    """emitted: "all" rows are wanted, or a request's first 1 .. rows ("spread"), as an acceptance step leaves them."""
    return dict(op="logprobs", batch=batch, rows=rows, vocab=vocab, dtype=dtype, top=top, temperature=temperature,
                masked=masked, emitted=emitted)


def _fork(prompts, samples, hkv, page, lo, hi, pool):
    return dict(op="fork", prompts=prompts, samples=samples, hkv=hkv, page=page, lo=lo, hi=hi, pool=pool)


def _compact(rows, done, hkv, page, lo, hi, pool):
    return dict(op="compact", rows=rows, done=done, hkv=hkv, page=page, lo=lo, hi=hi, pool=pool)


def listed():
    return [
        # one interactive request, a token at a time: latency
        dict(name="attn-b1-decode", **_attn(1, 1, 32, 8, 16, "const", 512, 512)),
        # parallel serving with short drafts: ragged contexts, seven query heads a KV head
        dict(name="attn-b64-ragged", **_attn(64, 5, 28, 4, 16, "lognormal", 512, 8192)),
        # a full server without drafts: the cache's bytes and little else
        dict(name="attn-b256-decode", **_attn(256, 1, 32, 8, 16, "uniform", 1024, 8192)),
        # a full server with drafts of eight over long contexts: the largest call
        dict(name="attn-b256-long", **_attn(256, 9, 64, 8, 32, "uniform", 2048, 16384)),
        # the rows of a verify step
        dict(name="append-step", **_append(64, 5, 4, 16, 512, 8192)),
        # the prompts of a burst of requests
        dict(name="append-prompts", **_append(16, 2049, 8, 16, 2049, 4096)),
        # one request of a small model under a grammar that masks half of its (odd) vocabulary
        dict(name="logprobs-b1", **_logprobs(1, 1, 32001, "f32", 5, 1.0, 0.5, "all")),
        # the emitted tokens of a full server's acceptance step
        dict(name="logprobs-b256", **_logprobs(256, 9, 128256, "bf16", 20, 0.8, 0.0, "spread")),
        # four samples of one prompt
        dict(name="fork-p1", **_fork(1, 4, 8, 16, 1000, 1000, "packed")),
        # a batch of prompts, three samples each
        dict(name="fork-p64", **_fork(64, 3, 8, 16, 1024, 16384, "bf16")),
        # a small server's pool after one request in three has finished
        dict(name="compact-b8", **_compact(8, 0.34, 8, 16, 512, 2048, "bf16")),
        # a full server's, after half of them
        dict(name="compact-b256", **_compact(256, 0.5, 8, 16, 1024, 8192, "packed")),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(("attn", "attn", "attn", "append", "logprobs", "logprobs", "fork", "compact"))
    page = rng.choice((16, 16, 32, 64))
    hq, hkv = rng.choice(_HEADS)
    while op == "attn":
        rows, batch, lo = _log_int(rng, 1, 17), _log_int(rng, 1, 256), _log_int(rng, 64, 8192)
        hi = _log_int(rng, lo, 16384)
        c = _attn(batch, rows, hq, hkv, page, "uniform", lo, hi)
        # at most the keys, scores and query rows of the largest listed case
        if (rows * (hq // hkv) <= 144 and lo > rows and batch * hkv * hi <= 256 * 8 * 16384
                and batch * rows * hq * hi <= 256 * 9 * 64 * 16384):
            return c
    while op == "append":
        n, batch, lo = _log_int(rng, 1, 4096), _log_int(rng, 1, 256), _log_int(rng, 64, 8192)
        hi = _log_int(rng, lo, 8192)
        if lo >= n and batch * hi * hkv <= 1 << 23:
            return _append(batch, n, hkv, page, lo, hi)
    while op == "logprobs":
        batch, rows = _log_int(rng, 1, 512), _log_int(rng, 1, 17)
        vocab = rng.choice(_VOCABS) if rng.random() < 0.4 else _log_int(rng, 8000, 256000)
        if batch * rows * vocab <= 256 * 9 * 128256:
            return _logprobs(batch, rows, vocab, "f32" if rng.random() < 0.3 else "bf16",
                             rng.choice((0, 1, 5, 8, 20)), round(rng.uniform(0.5, 1.2), 3),
                             rng.choice((0.0, 0.0, 0.3, 0.9)), rng.choice(("all", "spread")))
    pool = rng.choice(("packed", "bf16"))
    while True:
        lo = _log_int(rng, 64, 8192)
        hi = _log_int(rng, lo, 16384)
        if op == "fork":
            prompts, samples = _log_int(rng, 1, 64), _log_int(rng, 1, 8)
            if prompts * (hi + samples * page) * hkv <= 64 * 8 * 16384:
                return _fork(prompts, samples, hkv, page, lo, hi, pool)
        else:
            rows = _log_int(rng, 2, 256)
            if rows * hi * hkv * (1 if pool == "packed" else 3.5) <= 256 * 8 * 8192:
                return _compact(rows, round(rng.uniform(0.1, 0.9), 2), hkv, page, lo, hi, pool)


# --------------------------------------------------------------------------
# the packed format
# --------------------------------------------------------------------------
def _quantise(x, head):
    """Codes (two dims a byte, the even one low) and e4m3 scales of rows x [..., H, D]; head: fp32 [H]."""
    g = x.float().unflatten(-1, (D // GROUP, GROUP))
    s = (g.abs().amax(-1) / (6.0 * head[:, None])).clamp(max=448.0).to(torch.float8_e4m3fn)
    unit = (s.float() * head[:, None])[..., None]
    q = torch.where(unit > 0, g / unit, torch.zeros_like(g))
    a = q.abs()
    # nearest, ties to the even code
    code = ((a > 0.25).byte() + (a >= 0.75) + (a > 1.25) + (a >= 1.75) + (a > 2.5) + (a >= 3.5) + (a > 5.0)
            + 8 * torch.signbit(q)).byte().flatten(-2)
    return code[..., 0::2] | (code[..., 1::2] << 4), s


def _dequantise(codes, scales, head):
    """fp32 rows [..., H, n, D] of codes [..., H, n, D / 2] (and so on), H the third dim from the end."""
    one = torch.tensor(E2M1 + tuple(-v for v in E2M1), dtype=torch.float32, device=codes.device)
    byte = torch.arange(256, device=codes.device)
    both = torch.stack((one[byte & 15], one[byte >> 4]), dim=1)
    x = both[codes.int()].flatten(-2).unflatten(-1, (D // GROUP, GROUP))
    return (x * (scales.float() * head[:, None, None])[..., None]).flatten(-2)


def _random_pool(pages, hkv, page, gen):
    """A pool of quantised N(0, 1) keys and values, heads of different sizes."""
    out = []
    for _ in range(2):
        head = 2.0 ** (torch.rand(hkv, generator=gen, device=DEVICE) * 2 - 1)
        codes = torch.empty((pages, hkv, page, D // 2), dtype=torch.uint8, device=DEVICE)
        scales = torch.empty((pages, hkv, page, D // GROUP), dtype=torch.float8_e4m3fn, device=DEVICE)
        step = max(1, (1 << 27) // (hkv * page * D))
        for p in range(0, pages, step):
            n = min(step, pages - p)
            x = torch.randn((n, page, hkv, D), generator=gen, device=DEVICE) * head[:, None] / 2
            c, s = _quantise(x, head / 8)
            codes[p:p + n], scales[p:p + n] = c.transpose(1, 2), s.transpose(1, 2)
        out.append((codes, scales, head / 8))
    (kc, ks, kh), (vc, vs, vh) = out
    return kc, ks, vc, vs, kh, vh


# --------------------------------------------------------------------------
# inputs
# --------------------------------------------------------------------------
def _lens(case, n, gen, least):
    lo, hi = max(case["lo"], least), case["hi"]
    if case.get("ctx") == "lognormal":
        z = torch.randn(n, generator=gen, device=DEVICE)
        return torch.exp(math.log(2048) + 0.6 * z).round().clamp(lo, hi).int()
    return torch.randint(lo, hi + 1, (n,), generator=gen, device=DEVICE).int()


def _tables(lens, max_pages, page, pages, gen):
    """A page table of rows whose pages lie anywhere in the pool, -1 past each row's last."""
    order = torch.randperm(pages, generator=gen, device=DEVICE).int()
    need = (lens + page - 1) // page
    col = torch.arange(max_pages, device=DEVICE)[None]
    at = (torch.cumsum(need, 0) - need)[:, None] + col
    held = col < need[:, None]
    return torch.where(held, order[at.clamp(max=pages - 1)], torch.full_like(held, -1, dtype=torch.int32)).contiguous()


def _counts(table, pages):
    refs = torch.zeros(pages + 1, dtype=torch.int32, device=DEVICE)
    refs.index_add_(0, torch.where(table < 0, pages, table).flatten(), torch.ones_like(table).flatten())
    return refs[:pages].contiguous()


def _plain_pool(pages, hkv, page, gen, kind):
    """The pool's tensors, each [pages, ...]: bf16 keys and values, or codes and scales."""
    if kind == "bf16":
        return [torch.empty((pages, hkv, page, D), dtype=torch.bfloat16, device=DEVICE).normal_(generator=gen)
                for _ in range(2)]
    byte = lambda w: torch.randint(0, 120, (pages, hkv, page, w), generator=gen, device=DEVICE, dtype=torch.uint8)  # noqa: E731
    return [byte(D // 2), byte(D // GROUP), byte(D // 2), byte(D // GROUP)]


def prepare(case, seed):
    gen = torch.Generator(device=DEVICE).manual_seed(seed)
    op, s = case["op"], dict(case=case)
    if op == "logprobs":
        B, R, V = case["batch"], case["rows"], case["vocab"]
        dt = torch.float32 if case["dtype"] == "f32" else torch.bfloat16
        z = torch.empty((B * R, V), device=DEVICE).normal_(generator=gen).mul_(3.0)
        if case["masked"] > 0:
            z.masked_fill_(torch.rand((1, V), generator=gen, device=DEVICE) < case["masked"], -math.inf)
        s["logits"] = z.to(dt)
        tokens = (z - torch.empty_like(z).exponential_(generator=gen).log_().mul_(case["temperature"])).argmax(1)
        tokens = tokens.int().reshape(B, R)
        # a request emits 1 .. R tokens; -1 past them
        if case["emitted"] == "spread":
            n = 1 + torch.arange(B, device=DEVICE) * 5 % R
            tokens = torch.where(torch.arange(R, device=DEVICE)[None] < n[:, None], tokens, -1)
        s["tokens"] = tokens.reshape(-1).contiguous()
        return s
    page, hkv = case["page"], case["hkv"]
    max_pages = -(-case["hi"] // page)
    if op in ("attn", "append"):
        B = case["batch"]
        pages = B * max_pages
        s["lens"] = _lens(case, B, gen, case.get("rows", case.get("n_new")))
        s["table"] = _tables(s["lens"], max_pages, page, pages, gen)
        s["pool"] = _random_pool(pages, hkv, page, gen)
        if op == "attn":
            s["q"] = torch.randn((B, case["rows"], case["hq"], D), generator=gen, device=DEVICE).bfloat16()
        else:
            size = (s["pool"][4] * 4)[:, None], (s["pool"][5] * 4)[:, None]
            s["new"] = [(torch.randn((B, case["n_new"], hkv, D), generator=gen, device=DEVICE) * z).bfloat16()
                        for z in size]
        return s
    if op == "fork":
        n, k = case["prompts"], case["samples"]
        pages = n * max_pages + n * k
        lens = _lens(case, n, gen, 1)
        table = _tables(lens, max_pages, page, pages, gen)
        s["table"] = torch.cat((table, torch.full((n * k, max_pages), -1, dtype=torch.int32, device=DEVICE)))
        s["lens"] = torch.cat((lens, torch.zeros(n * k, dtype=torch.int32, device=DEVICE)))
        s["src"] = torch.arange(n, device=DEVICE).int().repeat_interleave(k)
        s["dst"] = torch.arange(n, n + n * k, device=DEVICE).int()
        s["zeros"] = torch.zeros_like(s["dst"])
    else:
        n = case["rows"]
        pages = n * max_pages
        s["lens"] = _lens(case, n, gen, 1)
        s["table"] = _tables(s["lens"], max_pages, page, pages, gen)
        s["done"] = torch.randperm(n, generator=gen, device=DEVICE)[:max(1, int(n * case["done"]))].int()
        s["zeros"] = torch.zeros_like(s["done"])
    s["refs"] = _counts(s["table"], pages)
    s["pools"] = _plain_pool(pages, hkv, page, gen, case["pool"])
    return s


# --------------------------------------------------------------------------
# one pass
# --------------------------------------------------------------------------
def run(state):
    return (_run_own if own else _run_plain)[state["case"]["op"]](state)


def _own_attn(s):
    from paper_2607_20507_gb300 import binding
    return dict(out=binding.cs_packed_verify_attention(s["q"], binding.PackedPool(*s["pool"]), s["table"], s["lens"],
                                                       s["case"]["rows"] - 1))


def _own_append(s):
    from paper_2607_20507_gb300 import binding
    pool = binding.PackedPool(*s["pool"])
    binding.cs_packed_kv_append(*s["new"], pool, s["table"], s["lens"])
    k, v = binding.cs_packed_kv_read(pool, s["table"], s["lens"], s["case"]["n_new"])
    return dict(k=k, v=v, k_scales=pool.k_scales, v_scales=pool.v_scales)


def _own_logprobs(s):
    from paper_2607_20507_gb300 import binding
    lp, entropy, top, top_lp = binding.cs_logprobs(s["logits"], s["tokens"], s["case"]["temperature"], s["case"]["top"])
    return dict(logprob=lp, entropy=entropy, top=top, top_logprob=top_lp)


def _own_fork(s):
    from paper_2607_20507_gb300 import binding
    page = s["case"]["page"]
    binding.cs_kv_release(s["table"], s["lens"], s["refs"], s["dst"], s["zeros"], page)
    done = binding.cs_kv_fork(s["pools"], s["table"], s["lens"], s["refs"], s["src"], s["dst"], page)
    return dict(forked=done, table=s["table"], lens=s["lens"], refs=s["refs"], pools=s["pools"])


def _own_compact(s):
    from paper_2607_20507_gb300 import binding
    # (the scheduler keeps this step's tables)
    table, lens, refs = s["table"].clone(), s["lens"].clone(), s["refs"].clone()
    binding.cs_kv_release(table, lens, refs, s["done"], s["zeros"], s["case"]["page"])
    live = binding.cs_kv_compact(s["pools"], table, refs)
    return dict(live=live, table=table, lens=lens, refs=refs, pools=s["pools"])


_run_own = dict(attn=_own_attn, append=_own_append, logprobs=_own_logprobs, fork=_own_fork, compact=_own_compact)


def _plain_attn(s):
    q, table, lens = s["q"], s["table"], s["lens"]
    kc, ks, vc, vs, kh, vh = s["pool"]
    B, R, hq, _ = q.shape
    hkv = kc.shape[1]
    at = table.clamp(min=0)
    dense = lambda c, z, h: _dequantise(c[at], z[at], h).transpose(1, 2).flatten(2, 3)  # noqa: E731  [B, H, L, D]
    x = q.float().unflatten(2, (hkv, hq // hkv)).permute(0, 2, 3, 1, 4).flatten(2, 3)   # [B, H, G R, D]
    score = x @ dense(kc, ks, kh).transpose(2, 3) / math.sqrt(D)
    last = lens[:, None] - R + torch.arange(R, device=q.device)[None]                   # row i's last key
    seen = torch.arange(score.shape[3], device=q.device)[None, None] <= last[:, :, None]
    score = score.unflatten(2, (-1, R)).masked_fill_(~seen[:, None, None], -math.inf).flatten(2, 3)
    p = torch.exp(score - score.amax(-1, keepdim=True))
    o = (p @ dense(vc, vs, vh)) / p.sum(-1, keepdim=True)
    return dict(out=o.unflatten(2, (-1, R)).permute(0, 3, 1, 2, 4).reshape(q.shape).bfloat16())


def _slots(table, lens, n, page):
    pos = lens[:, None].long() - n + torch.arange(n, device=lens.device)[None]
    return torch.gather(table, 1, pos // page).long(), pos % page


def _plain_append(s):
    kc, ks, vc, vs, kh, vh = s["pool"]
    page, slot = _slots(s["table"], s["lens"], s["case"]["n_new"], s["case"]["page"])
    for new, c, z, h in ((s["new"][0], kc, ks, kh), (s["new"][1], vc, vs, vh)):
        code, scale = _quantise(new, h)
        c[page, :, slot] = code
        z[page, :, slot] = scale
    row = lambda c, z, h: _dequantise(c[page, :, slot][..., None, :], z[page, :, slot][..., None, :],  # noqa: E731
                                      h).squeeze(-2).bfloat16()
    return dict(k=row(kc, ks, kh), v=row(vc, vs, vh), k_scales=ks, v_scales=vs)


def _plain_logprobs(s):
    T, n = s["case"]["temperature"], s["case"]["top"]
    z, tok = s["logits"].float(), s["tokens"].long()
    m = z.amax(1, keepdim=True)
    d = (z - m) / T
    w = torch.exp(d)
    total = w.sum(1)
    lse = torch.log(total)
    entropy = lse - torch.where(w > 0, w * d, torch.zeros_like(w)).sum(1) / total
    # the order of the logits, lowest id first on ties, as one whole number
    bits = (z + 0.0).view(torch.int32)
    key = (torch.where(bits < 0, bits ^ 0x7FFFFFFF, bits).long() << 32) - torch.arange(z.shape[1], device=z.device)[None]
    top = torch.topk(key, n, dim=1).indices
    top_lp = torch.gather(d, 1, top) - lse[:, None]
    lp = torch.gather(d, 1, tok.clamp(min=0)[:, None])[:, 0] - lse
    none, any_top = tok < 0, torch.isinf(top_lp)
    inf = torch.full_like(lp, -math.inf)
    return dict(logprob=torch.where(none, inf, lp), entropy=torch.where(none, torch.zeros_like(lp), entropy),
                top=torch.where(any_top | none[:, None], -1, top).int(),
                top_logprob=torch.where(none[:, None], inf[:, None], top_lp))


def _plain_release(table, lens, refs, rows, keep, page):
    r = rows.long()
    keep = torch.minimum(keep, lens[r])
    col = torch.arange(table.shape[1], device=table.device)[None]
    gone = (col >= ((keep + page - 1) // page)[:, None]) & (col < ((lens[r] + page - 1) // page)[:, None])
    old = table[r]
    refs.index_add_(0, old.clamp(min=0).flatten(), -gone.int().flatten())
    table[r] = torch.where(gone, -1, old)
    lens[r] = keep


def _plain_fork(s):
    table, lens, refs, page = s["table"], s["lens"], s["refs"], s["case"]["page"]
    _plain_release(table, lens, refs, s["dst"], s["zeros"], page)
    src, dst = s["src"].long(), s["dst"].long()
    L = lens[src]
    full, part = L // page, L % page > 0
    free = torch.cumsum((refs == 0).int(), 0)
    nth = torch.cumsum(part.int(), 0)
    done = ~part | (nth <= free[-1])
    fresh = torch.searchsorted(free, nth.clamp(max=free[-1])).int()
    old = table[src]
    col = torch.arange(table.shape[1], device=table.device)[None]
    shared = (col < full[:, None]) & done[:, None]
    refs.index_add_(0, old.clamp(min=0).flatten(), shared.int().flatten())
    table[dst] = torch.where(shared, old, torch.where((col == full[:, None]) & (part & done)[:, None], fresh[:, None], -1))
    lens[dst] = torch.where(done, L, 0)
    copies = torch.nonzero(part & done)[:, 0]
    to, of = fresh[copies].long(), torch.gather(old, 1, full.long()[:, None].clamp(max=table.shape[1] - 1))[copies, 0].long()
    refs[to] = 1
    for p in s["pools"]:
        p[to] = p[of]
    return dict(forked=done.int(), table=table, lens=lens, refs=refs, pools=s["pools"])


def _plain_compact(s):
    table, lens, refs = s["table"].clone(), s["lens"].clone(), s["refs"].clone()
    _plain_release(table, lens, refs, s["done"], s["zeros"], s["case"]["page"])
    live = refs > 0
    n = live.sum()
    ids = torch.arange(refs.shape[0], device=refs.device)
    of, to = torch.nonzero(live & (ids >= n))[:, 0], torch.nonzero(~live & (ids < n))[:, 0]
    where = ids.int()
    where[of] = to.int()
    refs[to] = refs[of]
    refs[of] = 0
    table = torch.where(table >= 0, where[table.clamp(min=0)], table)
    for p in s["pools"]:
        p[to] = p[of]
    return dict(live=n.int().reshape(1), table=table, lens=lens, refs=refs, pools=s["pools"])


_run_plain = dict(attn=_plain_attn, append=_plain_append, logprobs=_plain_logprobs, fork=_plain_fork,
                  compact=_plain_compact)


# --------------------------------------------------------------------------
# what a pass cannot do without
# --------------------------------------------------------------------------
def _mean(case):
    return 2048 * math.exp(0.18) if case.get("ctx") == "lognormal" else (case["lo"] + case["hi"]) / 2


def work(case):
    op = case["op"]
    row = D // 2 + D // GROUP        # one packed row of one head
    if op == "attn":
        B, L, R = case["batch"], _mean(case), case["rows"]
        return dict(bytes=B * (2 * L * case["hkv"] * row + 4 * R * case["hq"] * D + 4 * math.ceil(L / case["page"]) + 4),
                    flops=4 * B * R * case["hq"] * D * L)
    if op == "append":   # the rows in, their packed form out and in, the rows out
        n = 2 * case["batch"] * case["n_new"] * case["hkv"]
        return dict(bytes=n * (4 * D + 2 * row), flops=6 * n * D)
    if op == "logprobs":
        B, R, V, e = case["batch"], case["rows"], case["vocab"], 4 if case["dtype"] == "f32" else 2
        rows = B * R if case["emitted"] == "all" else sum(1 + b * 5 % R for b in range(B))
        return dict(bytes=rows * (V * e + 12 + 8 * case["top"]), flops=6 * rows * V)
    page_bytes = 2 * case["hkv"] * case["page"] * (2 * D if case["pool"] == "bf16" else row)
    pages = math.ceil(_mean(case) / case["page"])
    if op == "fork":     # part-filled pages in and out; counts and table entries of the shared ones, twice
        n = case["prompts"] * case["samples"]
        return dict(bytes=n * (2 * page_bytes + 24 * pages), flops=0)
    # the moved pages (of those in use, the share that lies past the new end) in and out, the table in and out
    spare = 1 - _mean(case) * (1 - case["done"]) / case["hi"]
    moved = case["rows"] * (1 - case["done"]) * pages * spare
    return dict(bytes=2 * moved * page_bytes + 8 * case["rows"] * math.ceil(case["hi"] / case["page"]), flops=0)


# --------------------------------------------------------------------------
# the results from the definitions in 64 bits
# --------------------------------------------------------------------------
_GRID = torch.tensor(E2M1, dtype=torch.float64)


def _values(codes, scales, head):
    """64-bit rows of packed [H, n, ...] and head scales [H]."""
    grid = _GRID.to(codes.device)
    lo, hi = codes & 15, codes >> 4
    v = torch.stack([grid[(c & 7).long()] * (1 - 2 * (c >> 3).double()) for c in (lo, hi)], -1).flatten(-2)
    return v * scales.double().repeat_interleave(GROUP, -1) * head.double()[:, None, None]


def _exact_attn(case, s):
    q = s["q"].double()
    kc, ks, vc, vs, kh, vh = s["pool"]
    R, hq, hkv = case["rows"], case["hq"], case["hkv"]
    out = torch.empty_like(q)
    for b, L in enumerate(s["lens"].tolist()):
        pages = s["table"][b, :-(-L // case["page"])].long()
        rows = lambda c, z, h: _values(c[pages].transpose(0, 1).flatten(1, 2)[:, :L],  # noqa: E731
                                       z[pages].transpose(0, 1).flatten(1, 2)[:, :L], h)
        x = q[b].unflatten(1, (hkv, hq // hkv))
        t = torch.einsum("rhgd,hld->hgrl", x, rows(kc, ks, kh)) / math.sqrt(D)
        causal = torch.ones((R, L), dtype=torch.bool, device=DEVICE).tril(L - R)
        p = torch.softmax(t.masked_fill(~causal, -math.inf), -1)
        out[b] = torch.einsum("hgrl,hld->rhgd", p, rows(vc, vs, vh)).flatten(1, 2)
    return dict(out=out)


def _e4m3(x):
    """The nearest e4m3 value (ties to even) of 0 <= x, at most 448."""
    step = torch.exp2(torch.floor(torch.log2(x.clamp(min=2.0 ** -6))) - 3)
    return (torch.round(x / step) * step).clamp(max=448.0)


def _exact_append(case, s):
    out = {}
    for name, new, head in (("k", s["new"][0], s["pool"][4]), ("v", s["new"][1], s["pool"][5])):
        h = head.double()[:, None, None]
        x = new.double().unflatten(-1, (D // GROUP, GROUP))
        scale = _e4m3(x.abs().amax(-1, keepdim=True) / (6 * h))
        unit = scale * h
        y = x / torch.where(unit > 0, unit, torch.ones_like(unit))
        a = y.abs().clamp(max=6.0)
        step = torch.where(a < 2, 0.5, torch.where(a < 4, 1.0, 2.0))
        out[name] = (torch.round(a / step) * step * torch.sign(y) * unit).flatten(-2)
    return dict(k=out["k"], v=out["v"], k_scales=None, v_scales=None)


def _exact_logprobs(case, s):
    z, tok = s["logits"], s["tokens"].long()
    out = dict(logprob=[], entropy=[], top_logprob=[])
    for r in range(0, z.shape[0], 64):
        lp = torch.log_softmax(z[r:r + 64].double() / case["temperature"], 1)
        t = tok[r:r + 64]
        none = t < 0
        out["logprob"].append(lp.gather(1, t.clamp(min=0)[:, None])[:, 0].masked_fill(none, -math.inf))
        out["entropy"].append(-torch.special.xlogy(lp.exp(), lp.exp()).sum(1).masked_fill(none, 0.0))
        out["top_logprob"].append(torch.topk(lp, case["top"], dim=1).values.masked_fill(none[:, None], -math.inf))
    return dict({k: torch.cat(v) for k, v in out.items()}, top=None)


def exact(case, seed):
    if case["op"] in ("fork", "compact"):
        return None   # pages, counts and tables: whole numbers and copies
    return dict(attn=_exact_attn, append=_exact_append, logprobs=_exact_logprobs)[case["op"]](case, prepare(case, seed))
