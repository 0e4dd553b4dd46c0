"""Rotated appends and chunk attention as a server uses them: prompts in chunks beside
requests that decode, both caches, the calls' marshalling, streams and capture."""
import numpy as np
import pytest
import torch

import ragged_reference as ref
import serving_reference as packed
from paper_2607_20507_gb300 import binding
from test_gpu_rope import table_of_turns

pytestmark = pytest.mark.gpu

DEV = "cuda:0"


def model(lengths, hq, hkv, ps, seed=0, fused=True):
    """Every request's projected tokens, a page table of whole rows and empty pools."""
    gen = torch.Generator(device=DEV).manual_seed(seed)
    B, cols = len(lengths), -(-max(lengths) // ps)
    P = B * cols + 1
    rows = [torch.randn((n, hq + 2 * hkv, 128), generator=gen, device=DEV).bfloat16() for n in lengths]
    table = torch.randperm(P, generator=torch.Generator().manual_seed(seed))[:B * cols].reshape(B, cols).int().to(DEV)
    norms = [(1 + 0.2 * torch.randn(128, generator=gen, device=DEV)).bfloat16() for _ in range(2)]
    return rows, table, P, norms, table_of_turns(cols * ps, 128)


def steps(rows, sizes):
    """The batches of a schedule: sizes[s][b] tokens of request b in step s; (tokens of all, lens, starts, counts)."""
    at = [0] * len(rows)
    for size in sizes:
        parts, lens, starts = [], [], [0]
        for b, n in enumerate(size):
            parts.append(rows[b][at[b]:at[b] + n])
            at[b] += n
            lens.append(at[b])
            starts.append(starts[-1] + n)
        yield (torch.cat(parts), torch.tensor(lens, dtype=torch.int32, device=DEV),
               torch.tensor(starts, dtype=torch.int32, device=DEV), size)


SCHEDULE = [(300, 1, 0, 77), (212, 1, 64, 1), (1, 1, 0, 1), (1, 130, 300, 1), (0, 1, 1, 20), (1, 1, 1, 1)]
LENGTHS = [sum(s[b] for s in SCHEDULE) for b in range(4)]


@pytest.mark.parametrize("hq,hkv,ps", [(8, 2, 16), (7, 1, 32), (4, 4, 8)])
def test_chunks_of_prompts_beside_requests_that_decode(hq, hkv, ps):
    rows, table, P, norms, turns = model(LENGTHS, hq, hkv, ps)
    pools = [torch.zeros((P, hkv, ps, 128), dtype=torch.bfloat16, device=DEV) for _ in range(2)]
    split = lambda x: (x[:, :hq], x[:, hq:hq + hkv], x[:, hq + hkv:])  # noqa: E731
    answers = [[] for _ in LENGTHS]
    for x, lens, starts, size in steps(rows, SCHEDULE):
        q = binding.cs_rope_kv_append(*split(x), turns, *pools, table, lens, starts, q_norm=norms[0], k_norm=norms[1])
        out = binding.cs_chunk_attention(q, *pools, table, lens, starts)
        expect, s = ref.attention(q, *pools, table, lens, starts)
        tol = 1.01 * 2.0 ** -8 * expect.abs() + (1.01 * 2.0 ** -8 + 2.0 ** -13) * s + 1e-37
        assert ((out.double() - expect).abs() <= tol).all()
        for b, o in enumerate(out.split(list(size))):
            answers[b].append(o)
    # the whole prompts at once: the same cache, and outputs that differ by roundings
    whole = [torch.zeros_like(p) for p in pools]
    x = torch.cat(rows)
    lens = torch.tensor(LENGTHS, dtype=torch.int32, device=DEV)
    starts = torch.zeros(5, dtype=torch.int32, device=DEV)
    starts[1:] = lens.cumsum(0)
    q = binding.cs_rope_kv_append(*split(x), turns, *whole, table, lens, starts, q_norm=norms[0], k_norm=norms[1])
    assert all(torch.equal(a, b) for a, b in zip(pools, whole))
    once = binding.cs_chunk_attention(q, *whole, table, lens, starts)
    _, s = ref.attention(q, *whole, table, lens, starts)
    pieces = torch.cat([torch.cat(a) for a in answers])
    assert ((once.double() - pieces.double()).abs() <= 1.01 * 2.0 ** -7 * once.double().abs() + 1.01 * 2.0 ** -7 * s).all()


def test_a_verify_step_on_the_cache_that_they_fill():
    """Prompts by chunk attention, then drafts by verify attention: as if the drafts were a chunk."""
    rows, table, P, norms, turns = model([205, 33, 1029], 16, 4, 16)
    pools = [torch.zeros((P, 4, 16, 128), dtype=torch.bfloat16, device=DEV) for _ in range(2)]
    for x, lens, starts, size in steps(rows, [(200, 28, 1024), (5, 5, 5)]):
        q = binding.cs_rope_kv_append(x[:, :16], x[:, 16:20], x[:, 20:], turns, *pools, table, lens, starts)
    out = binding.cs_chunk_attention(q, *pools, table, lens, starts)
    verified = binding.cs_verify_attention(q.reshape(3, 5, 16, 128), *pools, table, lens, 4).flatten(0, 1)
    _, s = ref.attention(q, *pools, table, lens, starts)
    assert ((out.double() - verified.double()).abs() <= 1.01 * 2.0 ** -7 * out.double().abs() + (2.0 ** -8 + 2.0 ** -12) * s).all()


def test_the_packed_cache():
    rows, table, P, norms, turns = model([70, 300, 5], 8, 2, 16)
    pool = binding.packed_pool(P, 2, 16, DEV)
    for x, lens, starts, size in steps(rows, [(69, 200, 0), (0, 99, 4), (1, 1, 1)]):
        q = binding.cs_packed_rope_kv_append(x[:, :8], x[:, 8:10], x[:, 10:], turns, pool, table, lens, starts,
                                             q_norm=norms[0], k_norm=norms[1])
    out = binding.cs_packed_verify_attention(q[:, None], pool, table, lens, 0)
    k, v = (packed.values(c.cpu().numpy(), s.cpu().view(torch.uint8).numpy(), np.ones(2))
            for c, s in ((pool.k_codes, pool.k_scales), (pool.v_codes, pool.v_scales)))
    expect, size = packed.packed_attention(q[:, None].double().cpu().numpy(), k, v, table.cpu().numpy(), lens.cpu().numpy(),
                                           128 ** -0.5)
    assert (np.abs(out.double().cpu().numpy() - expect) <= 1.01 * 2.0 ** -8 * np.abs(expect) + (2.0 ** -11 + 2.0 ** -15) * size + 1e-37).all()


class Interpreted:
    """In the place of the compiled marshalling: every call goes through the checks in Python."""
    def __getattr__(self, name):
        return lambda *a: None


def calls():
    rows, table, P, norms, turns = model([40, 90], 8, 2, 16, seed=5)
    x, lens, starts, _ = next(steps(rows, [(40, 90)]))
    pools = [torch.randn((P, 2, 16, 128), device=DEV).bfloat16() for _ in range(2)]
    return dict(q=x[:, :8], new_k=x[:, 8:10], new_v=x[:, 10:], cos_sin=turns, k_pages=pools[0], v_pages=pools[1],
                page_table=table, ctx_lens=lens, q_starts=starts), norms, P


def attend(a, **kw):
    a = {**a, **kw}
    return binding.cs_chunk_attention(a["q"], a["k_pages"], a["v_pages"], a["page_table"], a["ctx_lens"], a["q_starts"])


def append(a, **kw):
    return binding.cs_rope_kv_append(**{**a, **kw})


def append_packed(a, pool, **kw):
    b = {k: v for k, v in {**a, **kw}.items() if k not in ("k_pages", "v_pages")}
    return binding.cs_packed_rope_kv_append(pool=pool, **b)


def test_marshalling_does_what_the_checks_do(monkeypatch):
    a, norms, P = calls()

    def everything():
        pool = binding.packed_pool(P, 2, 16, DEV)
        b = {**a, "k_pages": a["k_pages"].clone(), "v_pages": a["v_pages"].clone()}
        out = [append(b, q_norm=norms[0], interleaved=True, norm_eps=1e-5), append_packed(b, pool, k_norm=norms[1])]
        assert append(b, q=None) is None and append_packed(b, pool, q=None) is None
        q_out = torch.zeros_like(a["q"])
        assert append(b, q_out=q_out) is q_out
        given = torch.zeros((130, 8, 128), dtype=torch.bfloat16, device=DEV)
        assert binding.cs_chunk_attention(a["q"], b["k_pages"], b["v_pages"], a["page_table"], a["ctx_lens"], a["q_starts"],
                                          out=given, sm_scale=0.2) is given
        return out + [q_out, given, attend(b), b["k_pages"], b["v_pages"], *(t.view(torch.uint8) for t in pool[:4])]

    fast = everything()
    binding._load_fast()
    monkeypatch.setattr(binding, "_fast", Interpreted())
    for x, y in zip(fast, everything()):
        assert torch.equal(x.contiguous(), y.contiguous())


BAD = [
    (dict(q=lambda t: t.float()), TypeError), (dict(q=lambda t: t.cpu()), ValueError), (dict(q=lambda t: t[:, :, :64]), ValueError),
    (dict(q=lambda t: t[0]), ValueError), (dict(q=lambda t: t.transpose(0, 1)), ValueError),
    (dict(q=lambda t: t.expand(130, 8, 128) if t.shape[0] == 1 else t[:1].expand(130, 8, 128)), ValueError),
    (dict(q=lambda t: torch.empty((130, 9, 132), device=DEV, dtype=torch.bfloat16)[:, :8, :128]), ValueError),
    (dict(k_pages=lambda t: t.transpose(1, 2)), ValueError), (dict(v_pages=lambda t: t[:-1].contiguous()), ValueError),
    (dict(page_table=lambda t: t.long()), TypeError), (dict(page_table=lambda t: t[:1].contiguous()), ValueError),
    (dict(ctx_lens=lambda t: t.float()), TypeError), (dict(ctx_lens=lambda t: t.cpu()), ValueError),
    (dict(q_starts=lambda t: t[:2].contiguous()), ValueError), (dict(q_starts=lambda t: t.long()), TypeError),
]
MORE = [
    (dict(new_k=lambda t: t.half()), TypeError), (dict(new_k=lambda t: t[:-1]), ValueError),
    (dict(new_v=lambda t: t[:, :1]), ValueError), (dict(cos_sin=lambda t: t.double()), TypeError),
    (dict(cos_sin=lambda t: t[:, :100]), ValueError), (dict(q=lambda t: t[:-1]), ValueError),
]


def refused(call, a, change, error):
    wrong = {k: f(a[k]) for k, f in change.items()}
    with pytest.raises(error):
        call(a, **wrong)


@pytest.mark.parametrize("change,error", BAD)
def test_attention_refuses(change, error):
    refused(attend, calls()[0], change, error)


@pytest.mark.parametrize("change,error", [c for c in BAD if "v_pages" not in c[0]] + MORE)
def test_appends_refuse(change, error):
    a, _, P = calls()
    refused(append, a, change, error)
    if "k_pages" not in change:
        pool = binding.packed_pool(P, 2, 16, DEV)
        refused(lambda b, **kw: append_packed(b, pool, **kw), a, change, error)


def test_refusals_of_the_library_and_of_options():
    a, norms, P = calls()
    with pytest.raises(ValueError, match="without q_starts"):
        attend({**a, "page_table": a["page_table"].repeat(2, 1)[:3].contiguous(),
                "ctx_lens": torch.ones(3, dtype=torch.int32, device=DEV)}, q_starts=None)
    with pytest.raises(binding.CacheSpecError) as e:
        append(a, cos_sin=torch.zeros((48, 80), device=DEV))
    assert e.value.status == binding.CS_ERR_UNSUPPORTED
    with pytest.raises(binding.CacheSpecError) as e:
        append(a, norm_eps=-1.0)
    assert e.value.status == binding.CS_ERR_INVALID_ARG
    with pytest.raises(ValueError, match="positions"):
        append(a, positions=torch.zeros(4, dtype=torch.int32, device=DEV))
    with pytest.raises(ValueError, match="q_norm"):
        append(a, q_norm=norms[0][:64].contiguous())
    with pytest.raises(TypeError, match="k_norm"):
        append(a, k_norm=norms[0].float())
    with pytest.raises(ValueError, match="q_out"):
        append(a, q=None, q_out=torch.zeros((130, 8, 128), dtype=torch.bfloat16, device=DEV))
    with pytest.raises(binding.CacheSpecError) as e:
        binding.cs_chunk_attention(a["q"], a["k_pages"], a["v_pages"], a["page_table"], a["ctx_lens"], a["q_starts"],
                                   workspace=torch.zeros(256, dtype=torch.uint8, device=DEV))
    assert e.value.status == binding.CS_ERR_WORKSPACE


def test_a_step_on_another_stream_and_in_a_graph():
    """Append, attend, on a stream given by its handle; then captured, and replayed for the next step."""
    rows, table, P, norms, turns = model([400, 90], 8, 2, 16, seed=9)
    pools = [torch.zeros((P, 2, 16, 128), dtype=torch.bfloat16, device=DEV) for _ in range(2)]
    batches = list(steps(rows, [(300, 60), (3, 1), (3, 1)]))
    x, lens, starts, _ = batches[0]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    h = side.cuda_stream
    q = binding.cs_rope_kv_append(x[:, :8], x[:, 8:10], x[:, 10:], turns, *pools, table, lens, starts, stream=h)
    out = binding.cs_chunk_attention(q, *pools, table, lens, starts, stream=h)
    side.synchronize()
    expect, s = ref.attention(q, *pools, table, lens, starts)
    assert ((out.double() - expect).abs() <= 1.01 * 2.0 ** -8 * expect.abs() + (1.01 * 2.0 ** -8 + 2.0 ** -13) * s).all()
    x, lens, starts, _ = (t.clone() if torch.is_tensor(t) else t for t in batches[1])
    step = lambda: binding.cs_chunk_attention(  # noqa: E731
        binding.cs_rope_kv_append(x[:, :8], x[:, 8:10], x[:, 10:], turns, *pools, table, lens, starts), *pools, table, lens, starts)
    with torch.cuda.stream(side):
        step()
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        captured = step()
    for b in (1, 2):
        for old, new in zip((x, lens, starts), batches[b]):
            old.copy_(new)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(captured, step())
