"""The packed cache, page and log-probability calls as a server uses them: the example's loop, the compiled
marshalling against the interpreted checks, streams and given workspaces."""
import ctypes
import importlib.util
import os

import numpy as np
import pytest
import torch

from paper_2607_20507_gb300 import binding as b
from test_gpu_binding import both_ways

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def example():
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "packed_serving.py")
    spec = importlib.util.spec_from_file_location("packed_serving", path)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def counted(table, P):
    t = table.cpu().numpy()
    return np.bincount(t[(t >= 0) & (t < P)], minlength=P)


def held(pool, row, L):
    """What the cache holds for a row's first L tokens: (k, v), [L, Hkv, 128]."""
    return [x[0] for x in b.cs_packed_kv_read(pool, row, torch.tensor([L], dtype=torch.int32, device=DEV), L)]


@pytest.mark.parametrize("prompt", [1, 16, 333, 4101])
def test_example_loop(prompt):
    """After every call the counts are the table's entries; a row attends over what the cache holds for it; the log
    probabilities are those of the logits; what a row holds survives release and compaction."""
    ex = example()
    model = ex.StandIn(2, 8, 2, 3001, torch.device(DEV), seed=prompt)
    n, k, room = 3, 4, 40
    ps, cols = 16, (prompt + room) // 16 + 2
    s = ex.Server(model, 1 + n, cols + n * (room // ps + 2), ps, cols)
    P = s.counts.shape[0]
    assert s.prefill(0, prompt).all() and s.fork([0] * n, range(1, 1 + n), room).all()
    assert np.array_equal(s.counts.cpu().numpy(), counted(s.table, P))
    assert s.lens.tolist() == [prompt] * (1 + n)
    for _ in range(3):
        before = s.lens[1:].clone()
        out, acc, (lp, ent, top, top_lp) = s.step((1, 1 + n), k, 0.8, 3)
        assert torch.equal(s.lens[1:], before + 1 + acc)
        # the last layer's attention: its keys and values as the cache gives them
        q, pool, got = s.attended
        L = (before + k + 1).tolist()
        for r in range(n):
            K, V = (x.double() for x in held(pool, s.table[1 + r:2 + r], L[r]))
            z = torch.einsum("ihgd,jhd->ihgj", q[r].double().view(k + 1, 2, 4, 128), K) / 128 ** 0.5
            seen = torch.arange(L[r], device=DEV)[None, :] <= L[r] - k - 1 + torch.arange(k + 1, device=DEV)[:, None]
            p = z.masked_fill(~seen[:, None, None], -float("inf")).softmax(-1)
            want = torch.einsum("ihgj,jhd->ihgd", p, V).reshape(k + 1, 8, 128)
            # bf16 output (2^-8 of it), P in 11 bits (2^-11 of the mean of |V|) and the rows read rounded
            # to bf16 (no head scale: code * s has at most 6 bits, so they are exact), fp32 sums
            room_p = torch.einsum("ihgj,jhd->ihgd", p, V.abs()).reshape(k + 1, 8, 128) * 2 ** -10
            assert ((got[r].double() - want).abs() <= want.abs() * 2 ** -8 + room_p + 1e-5).all()
        z = (s.logits.double() / 0.8).view(-1, 3001).log_softmax(-1)
        on = out.view(-1) >= 0
        want = z.gather(1, out.view(-1, 1).clamp(min=0).long())[:, 0]
        assert torch.equal(on, torch.isfinite(lp)) and (lp.double() - want)[on].abs().max() < 1e-5
        assert (ent.double() + (z.exp() * z).sum(-1))[on].abs().max() < 1e-4
        order = torch.sort(s.logits.view(-1, 3001).float(), dim=-1, descending=True, stable=True).indices[:, :3]
        assert torch.equal(top[on].long(), order[on])
    before = [held(p, s.table[2:3], int(s.lens[2])) for p in s.pools]
    s.release([0, 1, 3])
    assert np.array_equal(s.counts.cpu().numpy(), counted(s.table, P))
    live = int(s.compact())
    assert np.array_equal(s.counts.cpu().numpy(), counted(s.table, P))
    assert live == int((s.counts > 0).sum()) and int(s.table.max()) == live - 1
    for p, old in zip(s.pools, before):
        for x, y in zip(held(p, s.table[2:3], int(s.lens[2])), old):
            assert torch.equal(x, y)


def test_example_runs(capsys):
    server, best = example().main(["--samples", "3", "--steps", "2", "--prompt", "50"])
    assert "pages in use" in capsys.readouterr().out
    assert (server.lens > 0).tolist() == [i == 1 + best for i in range(4)]


def case(seed=0):
    rng = np.random.default_rng(seed)
    H, ps, P, B, cols, k = 2, 16, 40, 3, 6, 2
    g = torch.Generator(device=DEV).manual_seed(seed)

    def normal(*shape):
        return torch.randn(shape, generator=g, device=DEV).to(torch.bfloat16)

    pool = b.packed_pool(P, H, ps, DEV, torch.tensor([0.5, 2.0], device=DEV), torch.tensor([1.5, 1.0], device=DEV))
    table = torch.from_numpy(rng.permutation(P)[:B * cols].reshape(B, cols).astype(np.int32)).to(DEV)
    lens = torch.tensor([70, 3, 96], dtype=torch.int32, device=DEV)
    b.cs_packed_kv_append(normal(B, 96, H, 128), normal(B, 96, H, 128), pool, table, lens)
    counts = torch.zeros((P,), dtype=torch.int32, device=DEV)
    counts[table.view(-1).long()] = 1
    return dict(pool=pool, table=table, lens=lens, counts=counts, k=k, q=normal(B, k + 1, 8, 128),
                new=(normal(B, k + 1, H, 128), normal(B, k + 1, H, 128)), logits=normal(5, 1003),
                tokens=torch.tensor([1, -1, 1002, 1003, 0], dtype=torch.int32, device=DEV))


def ints(*x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def in_place(call, *written):
    """What a call writes into copies of its arguments, after what it returns."""
    def run():
        x = [t.clone() for t in written]
        r = call(*x)
        return (() if r is None else (r,)) + tuple(x)
    return run


def test_marshalling_does_what_the_checks_do(monkeypatch):
    c = case()
    pool, table, lens, counts, k, q, z, tok = (c[n] for n in ("pool", "table", "lens", "counts", "k", "q", "logits",
                                                              "tokens"))
    heads = pool[4:]
    wide = torch.zeros((5, 2000), dtype=torch.bfloat16, device=DEV)
    wide[:, :1003] = z
    ws = torch.zeros(1 << 22, dtype=torch.uint8, device=DEV)
    pages = list(pool[:4])
    good = [
        in_place(lambda a, s, v, t: b.cs_packed_kv_append(*c["new"], (a, s, v, t, *heads), table, lens), *pool[:4]),
        lambda: b.cs_packed_kv_read(pool, table, lens, 7),
        lambda: b.cs_packed_verify_attention(q, pool, table, lens, k),
        lambda: b.cs_packed_verify_attention(q, tuple(pool[:4]) + (None, None), table, lens, k, sm_scale=0.3),
        lambda: b.cs_packed_verify_attention(q[:, :1].contiguous(), pool, table, lens, 0, workspace=ws),
        in_place(lambda p, t, n, r: b.cs_kv_fork([p], t, n, r, ints(0, -1), ints(1, 2), 16, 9), pool[0], table, lens, counts),
        in_place(lambda t, n, r: b.cs_kv_fork([], t, n, r, ints(2), ints(0), 16, workspace=ws), table, lens, counts),
        in_place(lambda t, n, r: b.cs_kv_release(t, n, r, ints(1, 2), ints(0, 17), 16), table, lens, counts),
        in_place(lambda p, v, t, r: b.cs_kv_compact([p, v], t, r), pool[0], pool[3], table, counts),
        in_place(lambda t, r: b.cs_kv_compact((), t, r, workspace=ws), table, counts),
        lambda: b.cs_logprobs(z, tok), lambda: b.cs_logprobs(z, tok, 0.8, 5), lambda: b.cs_logprobs(z.float(), tok, 2, 1),
        lambda: b.cs_logprobs(wide[:, :1003], tok, 0.8, 5)]
    for i, call in enumerate(good):
        fast, slow = both_ways(monkeypatch, call)
        assert isinstance(fast, list) and isinstance(slow, list) and 0 < len(fast) == len(slow), (i, fast, slow)
        for x, y in zip(fast, slow):
            assert x.dtype == y.dtype and x.shape == y.shape and torch.equal(x.view(torch.uint8), y.view(torch.uint8)), i
    bad = [
        lambda: b.cs_packed_kv_append(c["new"][0].float(), c["new"][1], pool, table, lens),
        lambda: b.cs_packed_kv_append(c["new"][0], c["new"][1][:2].contiguous(), pool, table, lens),
        lambda: b.cs_packed_kv_append(*c["new"], pool[:3], table, lens),
        lambda: b.cs_packed_kv_append(*c["new"], pool, table.long(), lens),
        lambda: b.cs_packed_kv_read(pool, table, lens[:2].contiguous(), 3),
        lambda: b.cs_packed_kv_read(pool, table, lens, 0), lambda: b.cs_packed_kv_read(pool, table, lens, -1),
        lambda: b.cs_packed_verify_attention(q, pool, table, lens, 3),
        lambda: b.cs_packed_verify_attention(q.transpose(1, 2), pool, table, lens, k),
        lambda: b.cs_packed_verify_attention(q, pool._replace(v_codes=pool.v_codes[:9]), table, lens, k),
        lambda: b.cs_packed_verify_attention(q, pool._replace(k_scales=pool.k_scales.view(torch.uint8)), table, lens, k),
        lambda: b.cs_packed_verify_attention(q, pool._replace(k_head_scale=torch.ones(3, device=DEV)), table, lens, k),
        lambda: b.cs_packed_verify_attention(q, pool, table, lens, k, sm_scale=float("inf")),
        lambda: b.cs_packed_verify_attention(q, pool, table, lens, k, workspace=torch.zeros(16, dtype=torch.uint8, device=DEV)),
        lambda: b.cs_packed_verify_attention(q, pool, table, lens, k, out=q[:2].contiguous()),
        lambda: b.cs_kv_fork(pages, table, lens, counts, ints(0), ints(1, 2), 16),
        lambda: b.cs_kv_fork(pages, table, lens, counts, ints(0), ints(1), 0),
        lambda: b.cs_kv_fork(pages, table, lens, counts, ints(0), ints(1), 16, -1),
        lambda: b.cs_kv_fork([pool[0][:3]], table, lens, counts, ints(0), ints(1), 16),
        lambda: b.cs_kv_release(table, lens, counts, ints(0), ints(1, 2), 16),
        lambda: b.cs_kv_release(table, lens.cpu(), counts, ints(0), ints(1), 16),
        lambda: b.cs_kv_compact(pages, table, counts[:7].contiguous()),
        lambda: b.cs_kv_compact(pages, table[0], counts),
        lambda: b.cs_logprobs(z, tok[:4].contiguous()), lambda: b.cs_logprobs(z, tok.long()),
        lambda: b.cs_logprobs(z.half(), tok), lambda: b.cs_logprobs(z.t(), tok), lambda: b.cs_logprobs(z, tok, 0.0),
        lambda: b.cs_logprobs(z, tok, 1.0, 33), lambda: b.cs_logprobs(z, tok, 1.0, -1), lambda: b.cs_logprobs(z, tok, None)]
    for i, call in enumerate(bad):
        fast, slow = both_ways(monkeypatch, call)
        assert isinstance(fast, tuple) and fast == slow, (i, fast, slow)


def test_given_output_workspace_and_stream():
    c = case(1)
    args = (c["q"], c["pool"], c["table"], c["lens"], c["k"])
    expect, scores = b.cs_packed_verify_attention(*args), b.cs_logprobs(c["logits"], c["tokens"], 0.8, 4)
    d = b.AttnDims(3, 8, 2, 128, 16, 6, 40, 0.0)
    n = b.load_library().cs_packed_verify_attention_workspace_bytes(ctypes.byref(d), c["k"])
    ws = torch.full((n,), 0xA5, dtype=torch.uint8, device=DEV)      # any contents
    out, side = torch.empty_like(c["q"]), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    assert b.cs_packed_verify_attention(*args, out=out, workspace=ws, stream=side.cuda_stream) is out
    side.synchronize()
    assert torch.equal(out, expect) and b.cs_read_device_status(ws) == 0
    with torch.cuda.stream(side):
        again, lp = b.cs_packed_verify_attention(*args), b.cs_logprobs(c["logits"], c["tokens"], 0.8, 4)
    side.synchronize()
    assert torch.equal(again, expect) and all(torch.equal(x, y) for x, y in zip(lp, scores))


def test_captured_in_a_graph():
    """The step's calls replay: append, attend, score, commit, with the lengths on the device."""
    c = case(2)
    pool, table, lens, k = c["pool"], c["table"], c["lens"].clone(), c["k"]
    acc = ints(1, 0, 2)

    def step(lens):
        lens += k + 1
        b.cs_packed_kv_append(*c["new"], pool, table, lens)
        o = b.cs_packed_verify_attention(c["q"], pool, table, lens, k)
        b.cs_kv_commit(lens, acc, k)
        return o, b.cs_logprobs(c["logits"], c["tokens"], 0.8, 4)[0]

    kept = [t.clone() for t in pool[:4]]
    want = [step(lens) for _ in range(3)]
    for t, old in zip(pool[:4], kept):
        t.copy_(old)
    lens = c["lens"].clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        step(c["lens"].clone())        # workspaces made before the capture
    side.synchronize()
    for t, old in zip(pool[:4], kept):
        t.copy_(old)
    with torch.cuda.graph(graph, stream=side):
        o, lp = step(lens)
    lens.copy_(c["lens"])
    for w in want:
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(o, w[0]) and torch.equal(lp, w[1])
