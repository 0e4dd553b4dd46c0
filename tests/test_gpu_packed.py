"""The packed cache on the GPU: rows in (bytes), rows out, and verify attention
against the definition in 64 bits."""
import numpy as np
import pytest
import torch

import serving_reference as ref
from paper_2607_20507_gb300 import binding

pytestmark = pytest.mark.gpu

DEV = "cuda:0"


def host(t):
    return t.detach().cpu().view(torch.uint8).numpy() if t.dtype == torch.float8_e4m3fn else t.detach().cpu().numpy()


def random_pool(rng, P, H, ps, heads=True, junk=False):
    """A pool of random codes and of scales between 2^-4 and 8 (junk: any byte, NaN among them)."""
    t = []
    for _ in range(2):
        codes = rng.integers(0, 256, (P, H, ps, 64), dtype=np.uint8)
        scales = rng.integers(0, 256, (P, H, ps, 8), dtype=np.uint8) if junk else \
            rng.integers(0x18, 0x50, (P, H, ps, 8), dtype=np.uint8)
        t += [torch.from_numpy(codes).to(DEV), torch.from_numpy(scales).to(DEV).view(torch.float8_e4m3fn)]
    if heads:
        t += [torch.from_numpy((2.0 ** rng.uniform(-3, 1, H)).astype(np.float32)).to(DEV) for _ in range(2)]
    return binding.PackedPool(*t)


def head_of(pool, which, H):
    h = pool.k_head_scale if which == "k" else pool.v_head_scale
    return np.ones(H) if h is None else host(h).astype(np.float64)


def dense(pool):
    H = pool.k_codes.shape[1]
    return (ref.values(host(pool.k_codes), host(pool.k_scales), head_of(pool, "k", H)),
            ref.values(host(pool.v_codes), host(pool.v_scales), head_of(pool, "v", H)))


def table_of(rng, B, cols, P):
    return rng.permutation(P)[:B * cols].reshape(B, cols).astype(np.int32)


def check_attention(q, pool, table, lens, n_draft, kv=None, **kw):
    out = binding.cs_packed_verify_attention(q, pool, torch.from_numpy(table).to(DEV), torch.from_numpy(lens).to(DEV),
                                             n_draft, **kw)
    k, v = dense(pool) if kv is None else kv
    scale = kw.get("sm_scale", 0.0)
    expect, size = ref.packed_attention(q.double().cpu().numpy(), k, v, table, lens, scale if scale > 0 else 128 ** -0.5)
    got = out.double().cpu().numpy()
    # the output's rounding to bf16 (8 significant bits: 2^-8 of the value at most),
    # the weights' to fp16 (11 bits: 2^-11), and fp32 sums and exponents (scores up to
    # some hundreds: 2^-15)
    tol = 1.01 * 2.0 ** -8 * np.abs(expect) + (2.0 ** -11 + 2.0 ** -15) * size + 1e-37
    bad = ~(np.abs(got - expect) <= tol)
    assert not bad.any(), (int(bad.sum()), np.argwhere(bad)[:4], got[bad][:4], expect[bad][:4])
    return out


# ------------------------------------------------------------ rows in and out
@pytest.mark.parametrize("B,n,H,ps,cols", [(3, 5, 2, 16, 6), (1, 1, 1, 8, 3), (8, 6, 8, 32, 5), (2, 70, 4, 64, 2),
                                           (5, 1, 3, 128, 1), (2, 257, 1, 256, 2), (40, 3, 5, 8, 4)])
@pytest.mark.parametrize("heads", [False, True])
def test_append_is_the_definition(B, n, H, ps, cols, heads):
    rng = np.random.default_rng(B * 100 + n + ps)
    P = B * cols + 3
    pool = random_pool(rng, P, H, ps, heads)
    table, lens = table_of(rng, B, cols, P), rng.integers(0, cols * ps + 1, B).astype(np.int32)
    new = [torch.from_numpy((rng.standard_normal((B, n, H, 128)) * 2.0 ** rng.integers(-3, 4, (B, n, H, 1)))
                            .astype(np.float32)).bfloat16() for _ in range(2)]
    expect = [host(t).copy() for t in pool[:4]]
    for which, x, c, s in (("k", new[0], 0, 1), ("v", new[1], 2, 3)):
        codes, scales = ref.quantise(x.float().numpy(), head_of(pool, which, H))
        for b, i, page, slot in ref.place(table, lens, n, ps, P):
            expect[c][page, :, slot], expect[s][page, :, slot] = codes[b, i], scales[b, i]
    dt, dl = torch.from_numpy(table).to(DEV), torch.from_numpy(lens).to(DEV)
    binding.cs_packed_kv_append(new[0].to(DEV), new[1].to(DEV), pool, dt, dl)
    for t, e in zip(pool[:4], expect):
        np.testing.assert_array_equal(host(t), e)
    got = binding.cs_packed_kv_read(pool, dt, dl, n)
    for which, g, d in zip("kv", got, dense(pool)):
        want = np.zeros((B, n, H, 128))
        for b, i, page, slot in ref.place(table, lens, n, ps, P):
            want[b, i] = d[page, :, slot]
        # code * scale is exact; times the head's scale in fp32, then bf16
        np.testing.assert_allclose(g.double().cpu().numpy(), want, rtol=1.01 * 2.0 ** -8, atol=0)


def test_append_of_extreme_values():
    """Zeros, denormals, the type's largest, infinities, NaN, and every tie of the code grid."""
    H = 2
    rows = np.zeros((1, 12, H, 128), np.float32)
    rows[0, 1] = 1e-40
    rows[0, 2] = 3.3e38 * np.where(np.arange(128) % 2, 1, -1)
    rows[0, 3, :, ::7] = np.inf
    rows[0, 3, :, 3::16] = -np.inf
    rows[0, 4, :, ::5] = np.nan
    rows[0, 4, :, 1::5] = 2.0
    rows[0, 5] = np.nan
    ties = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0])
    for i, s in enumerate((1.0, 1.125, 0.8125, 448.0, 2.0 ** -9, 3 * 2.0 ** -9)):
        rows[0, 6 + i] = np.tile(np.concatenate((ties, -ties)) * s, 8)
    rows[0, 11, 1] = -0.0
    x = torch.from_numpy(rows).bfloat16()
    pool = binding.packed_pool(2, H, 16, DEV)
    table, lens = np.array([[1]], np.int32), np.array([12], np.int32)
    binding.cs_packed_kv_append(x.to(DEV), (-x).to(DEV), pool, torch.from_numpy(table).to(DEV),
                                torch.from_numpy(lens).to(DEV))
    for t, c, s in ((x, pool.k_codes, pool.k_scales), (-x, pool.v_codes, pool.v_scales)):
        codes, scales = ref.quantise(t.float().numpy(), np.ones(H))
        np.testing.assert_array_equal(host(s)[1, :, :12], scales[0].swapaxes(0, 1))
        np.testing.assert_array_equal(host(c)[1, :, :12], codes[0].swapaxes(0, 1))
    k, _ = binding.cs_packed_kv_read(pool, torch.from_numpy(table).to(DEV), torch.from_numpy(lens).to(DEV), 12)
    assert torch.isfinite(k).all()


def test_append_and_read_outside_the_pool():
    rng = np.random.default_rng(5)
    B, n, H, ps, cols, P = 6, 5, 2, 16, 3, 30
    pool = random_pool(rng, P, H, ps)
    table, lens = table_of(rng, B, cols, P), np.array([0, 2, -7, 10 ** 9, 20, 33], np.int32)
    table[4] = (-1, P, 1 << 30)
    new = torch.from_numpy(rng.standard_normal((B, n, H, 128)).astype(np.float32)).bfloat16()
    before = [host(t).copy() for t in pool[:4]]
    dt, dl = torch.from_numpy(table).to(DEV), torch.from_numpy(lens).to(DEV)
    binding.cs_packed_kv_append(new.to(DEV), new.to(DEV), pool, dt, dl)
    written = set((p, s) for _, _, p, s in ref.place(table, lens, n, ps, P))
    for t, b in zip(pool[:4], before):
        t = host(t)
        for p in range(P):
            for s in range(ps):
                if (p, s) not in written:
                    np.testing.assert_array_equal(t[p, :, s], b[p, :, s])
    k, v = binding.cs_packed_kv_read(pool, dt, dl, n)
    assert (k[2] == 0).all() and (v[0] == 0).all() and (k[4] == 0).all() and (k[1, :3] == 0).all()


def test_read_of_a_whole_context():
    rng = np.random.default_rng(6)
    pool = random_pool(rng, 9, 2, 64)
    table, lens = table_of(rng, 2, 4, 9), np.array([250, 7], np.int32)
    k, v = binding.cs_packed_kv_read(pool, torch.from_numpy(table).to(DEV), torch.from_numpy(lens).to(DEV), 256)
    for g, d in zip((k, v), dense(pool)):
        want = np.zeros((2, 256, 2, 128))
        for b, i, page, slot in ref.place(table, lens, 256, 64, 9):
            want[b, i] = d[page, :, slot]
        np.testing.assert_allclose(g.double().cpu().numpy(), want, rtol=1.01 * 2.0 ** -8, atol=0)


# ---------------------------------------------------------------- attention
@pytest.mark.parametrize("Hq,Hkv", [(32, 8), (28, 4), (64, 8), (4, 4), (40, 8), (3, 1), (16, 2)])
@pytest.mark.parametrize("k", [0, 1, 4, 8, 16])
def test_attention_heads_and_drafts(Hq, Hkv, k):
    if (k + 1) * (Hq // Hkv) > 144:
        pytest.skip("more query rows than a call takes")
    rng = np.random.default_rng(Hq * 31 + k)
    B, ps, cols = 3, 16, 20
    pool = random_pool(rng, B * cols, Hkv, ps)
    lens = rng.integers(k + 1, cols * ps + 1, B).astype(np.int32)
    q = torch.randn(B, k + 1, Hq, 128, generator=torch.Generator().manual_seed(k)).bfloat16().to(DEV)
    check_attention(q, pool, table_of(rng, B, cols, B * cols), lens, k)


@pytest.mark.parametrize("ps", [8, 16, 32, 64, 128, 256])
@pytest.mark.parametrize("rows,G", [(1, 4), (5, 7), (9, 8), (17, 8)])
def test_attention_pages_and_lengths(ps, rows, G):
    """Lengths around every edge: none, one, up to the draft, a page, a tile."""
    rng = np.random.default_rng(ps + rows)
    lens = np.array([0, 1, 2, rows - 1, rows, rows + 1, 15, 16, 17, 31, 33, 63, 64, 65, 127, 129, 255, 257, 512], np.int32)
    B, H = len(lens), 2
    cols = -(-512 // ps)
    P = B * cols
    pool = random_pool(rng, P, H, ps, heads=False)
    q = (torch.randn(B, rows, H * G, 128, generator=torch.Generator().manual_seed(ps)) * 0.3).bfloat16().to(DEV)
    out = check_attention(q, pool, table_of(rng, B, cols, P), lens, rows - 1)
    assert (out[0] == 0).all()                    # no key at all
    if rows > 2:
        assert (out[1, :rows - 1] == 0).all()     # one key: the last row's alone


def test_attention_many_ragged_requests():
    """More requests than a launch schedules at a time, most of them short."""
    rng = np.random.default_rng(11)
    B, ps, cols, P = 1100, 16, 10, 400
    lens = np.minimum(rng.geometric(0.02, B), cols * ps).astype(np.int32)
    lens[rng.integers(0, B, 40)] = 0
    table = rng.integers(0, P, (B, cols)).astype(np.int32)   # (pages shared by several rows)
    pool = random_pool(rng, P, 1, ps)
    q = torch.randn(B, 2, 3, 128, generator=torch.Generator().manual_seed(1)).bfloat16().to(DEV)
    check_attention(q, pool, table, lens, 1)


@pytest.mark.parametrize("rows,G,L", [(1, 8, 40000), (2, 4, 33001), (9, 8, 20011)])
def test_attention_one_long_request(rows, G, L):
    rng = np.random.default_rng(L)
    ps, H = 64, 1
    cols = -(-L // ps)
    pool = random_pool(rng, cols + 5, H, ps)
    q = torch.randn(1, rows, H * G, 128, generator=torch.Generator().manual_seed(2)).bfloat16().to(DEV)
    check_attention(q, pool, table_of(rng, 1, cols, cols + 5), np.array([L], np.int32), rows - 1)


def test_attention_pool_past_32_bits():
    """A pool of more than 2^32 bytes of codes; the pages in use lie at its end."""
    rng = np.random.default_rng(3)
    H, ps, cols = 8, 256, 2
    P = (1 << 32) // (H * ps * 64) + 40
    small = random_pool(rng, 2 * cols, H, ps, heads=False)
    big = binding.PackedPool(*(torch.zeros((P,) + t.shape[1:], dtype=torch.uint8, device=DEV).view(t.dtype)
                               for t in small[:4]))
    at = np.array([[P - 1, P - 7], [P - 3, P - 30]], np.int32)
    for s, t in zip(small[:4], big[:4]):
        t.view(torch.uint8)[torch.from_numpy(at.reshape(-1).astype(np.int64)).to(DEV)] = s.view(torch.uint8)
    lens = np.array([500, 257], np.int32)
    q = torch.randn(2, 3, 32, 128, generator=torch.Generator().manual_seed(9)).bfloat16().to(DEV)
    dq = check_attention(q, small, np.arange(4, dtype=np.int32).reshape(2, 2), lens, 2)
    got = binding.cs_packed_verify_attention(q, big, torch.from_numpy(at).to(DEV), torch.from_numpy(lens).to(DEV), 2)
    assert torch.equal(got, dq)
    new = torch.randn(2, 3, H, 128, generator=torch.Generator().manual_seed(8)).bfloat16().to(DEV)
    dt, dl = torch.from_numpy(at).to(DEV), torch.from_numpy(lens).to(DEV)
    binding.cs_packed_kv_append(new, new, big, dt, dl)
    k, v = binding.cs_packed_kv_read(big, dt, dl, 3)
    assert torch.equal(k, v) and (k - new).abs().max() <= new.abs().max() / 6 + 0.05


def test_attention_pages_outside_the_pool_read_as_zeros():
    rng = np.random.default_rng(12)
    B, ps, cols, P = 4, 16, 6, 24
    pool = random_pool(rng, P, 2, ps)
    table = table_of(rng, B, cols, P)
    table[1, 2], table[2] = P, (-1, -5, 1 << 30, P, P + 1, -(1 << 31))
    q = torch.randn(B, 3, 8, 128, generator=torch.Generator().manual_seed(3)).bfloat16().to(DEV)
    lens = np.array([96, 96, 90, 1 << 30], np.int32)
    out = check_attention(q, pool, table, lens, 2)
    assert (out[2] == 0).all()


@pytest.mark.parametrize("rows", [1, 4])
def test_attention_never_sees_slots_past_the_context(rows):
    """Every byte past L, NaN scales among them, and the pages past the last one."""
    rng = np.random.default_rng(13)
    B, ps, cols, H = 5, 32, 4, 2
    P = B * cols
    pool = random_pool(rng, P, H, ps)
    table = table_of(rng, B, cols, P)
    lens = np.array([4, 31, 33, 64, 101], np.int32)
    kv = dense(pool)
    for b in range(B):
        for pos in range(lens[b], cols * ps):
            for t in pool[:4]:
                t.view(torch.uint8)[table[b, pos // ps], :, pos % ps] = 0x7F
        table[b, -(-int(lens[b]) // ps):] = 1 << 29
    q = torch.randn(B, rows, 8, 128, generator=torch.Generator().manual_seed(4)).bfloat16().to(DEV)
    check_attention(q, pool, table, lens, rows - 1, kv=kv)


@pytest.mark.parametrize("size", [1e-30, 1e-6, 300.0, 3e4])
def test_attention_query_sizes(size):
    """Queries far from 1: fp16 would lose the first two and overflow at the last."""
    rng = np.random.default_rng(14)
    pool = random_pool(rng, 12, 2, 16, heads=False)
    q = (torch.randn(2, 3, 8, 128, generator=torch.Generator().manual_seed(5)) * size).bfloat16().to(DEV)
    check_attention(q, pool, table_of(rng, 2, 6, 12), np.array([96, 50], np.int32), 2, sm_scale=0.05 / size)


def test_attention_one_key_outweighs_the_rest():
    """A score hundreds above the others, early, late and in the middle of the context."""
    rng = np.random.default_rng(15)
    ps, cols, H = 16, 40, 1
    pool = random_pool(rng, 3 * cols, H, ps, heads=False)
    table = table_of(rng, 3, cols, 3 * cols)
    for b, pos in enumerate((0, 333, 638)):
        pool.k_codes[table[b, pos // ps], :, pos % ps] = 0x77
        pool.k_scales.view(torch.uint8)[table[b, pos // ps], :, pos % ps] = 0x58
    q = torch.rand(3, 2, 4, 128, generator=torch.Generator().manual_seed(6)).bfloat16().to(DEV)
    check_attention(q, pool, table, np.array([640, 640, 640], np.int32), 1)


def test_attention_same_bits_every_time_on_any_stream_and_workspace():
    rng = np.random.default_rng(16)
    B, ps, cols = 9, 16, 60
    pool = random_pool(rng, B * cols, 4, ps)
    table = torch.from_numpy(table_of(rng, B, cols, B * cols)).to(DEV)
    lens = torch.from_numpy(rng.integers(5, cols * ps + 1, B).astype(np.int32)).to(DEV)
    q = torch.randn(B, 5, 28, 128, generator=torch.Generator().manual_seed(7)).bfloat16().to(DEV)
    first = binding.cs_packed_verify_attention(q, pool, table, lens, 4)
    side = torch.cuda.Stream()
    for _ in range(3):
        assert torch.equal(first, binding.cs_packed_verify_attention(q, pool, table, lens, 4))
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        scaled = q * 1.0     # made on this stream, used on it
        again = binding.cs_packed_verify_attention(scaled, pool, table, lens, 4)
    side.synchronize()
    assert torch.equal(first, again)
    ws = torch.full((1 << 27,), 0xA5, dtype=torch.uint8, device=DEV)   # any contents
    assert torch.equal(first, binding.cs_packed_verify_attention(q, pool, table, lens, 4, workspace=ws))
    out = torch.empty_like(q)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        binding.cs_packed_verify_attention(q, pool, table, lens, 4, out=out)
    g.replay()
    torch.cuda.synchronize()
    assert torch.equal(first, out)


def test_attention_query_at_any_address():
    rng = np.random.default_rng(17)
    pool = random_pool(rng, 8, 2, 16)
    table = table_of(rng, 2, 4, 8)
    flat = torch.randn(2 * 3 * 8 * 128 + 2, generator=torch.Generator().manual_seed(8)).bfloat16().to(DEV)
    q = flat[2:].view(2, 3, 8, 128)
    assert q.data_ptr() % 16 == 4
    check_attention(q, pool, table, np.array([64, 33], np.int32), 2)


def test_append_read_and_attend():
    """A context appended in pieces reads like the rows themselves, to what 4 bits hold."""
    gen = torch.Generator().manual_seed(10)
    B, H, ps, cols = 2, 2, 16, 8
    pool = binding.packed_pool(B * cols, H, ps, DEV)
    table = torch.arange(B * cols, dtype=torch.int32, device=DEV).reshape(B, cols)
    lens = torch.zeros(B, dtype=torch.int32, device=DEV)
    rows = torch.randn(2, B, 100, H, 128, generator=gen).bfloat16().to(DEV)
    at = 0
    for n in (1, 40, 7, 52):
        lens += n
        binding.cs_packed_kv_append(*(r[:, at:at + n].contiguous() for r in rows), pool, table, lens)
        at += n
    k, v = binding.cs_packed_kv_read(pool, table, lens, 100)
    for got, want in ((k, rows[0]), (v, rows[1])):
        top = want.float().unflatten(-1, (8, 16)).abs().amax(-1, keepdim=True)
        # half the widest step (2 of 6), and the scale's rounding (2^-4)
        assert ((got - want).float().unflatten(-1, (8, 16)).abs() <= top * (1 / 6 + 1 / 16)).all()
    q = torch.randn(B, 1, 4, 128, generator=gen).bfloat16().to(DEV)
    out = binding.cs_packed_verify_attention(q, pool, table, lens, 0)
    s = torch.einsum("bhgd,blhd->bhgl", q[:, 0].double().unflatten(1, (H, 2)), k.double()) / 128 ** 0.5
    expect = torch.einsum("bhgl,blhd->bhgd", torch.softmax(s, -1), v.double()).flatten(1, 2)
    torch.testing.assert_close(out[:, 0].double(), expect, rtol=2.0 ** -8, atol=2.0 ** -9)


# ----------------------------------------------------------------- refusals
def test_binding_refuses():
    pool = binding.packed_pool(4, 2, 16, DEV)
    q = torch.zeros(1, 2, 4, 128, dtype=torch.bfloat16, device=DEV)
    table, lens = torch.zeros(1, 2, dtype=torch.int32, device=DEV), torch.ones(1, dtype=torch.int32, device=DEV)
    ok = lambda **k: binding.cs_packed_verify_attention(**{**dict(q=q, pool=pool, page_table=table, ctx_lens=lens,  # noqa: E731
                                                                  n_draft=1), **k})
    ok()
    with pytest.raises(ValueError):
        ok(n_draft=2)
    with pytest.raises(TypeError):
        ok(q=q.float())
    with pytest.raises(TypeError):
        ok(pool=pool._replace(k_scales=pool.k_scales.view(torch.uint8)))
    with pytest.raises(ValueError):
        ok(pool=pool._replace(v_codes=pool.v_codes[:3]))
    with pytest.raises(ValueError):
        ok(pool=pool._replace(k_head_scale=torch.ones(3, device=DEV)))
    with pytest.raises(ValueError):
        ok(pool=pool._replace(k_codes=pool.k_codes.transpose(1, 2)))
    with pytest.raises(ValueError):
        ok(page_table=table.repeat(2, 1))
    with pytest.raises(ValueError):
        ok(ctx_lens=lens.cpu())
    with pytest.raises(binding.CacheSpecError) as e:
        ok(workspace=torch.zeros(16, dtype=torch.uint8, device=DEV))
    assert e.value.status in (binding.CS_ERR_WORKSPACE, binding.CS_ERR_INVALID_ARG)
    new = torch.zeros(1, 1, 2, 128, dtype=torch.bfloat16, device=DEV)
    binding.cs_packed_kv_append(new, new, pool, table, lens)
    with pytest.raises(ValueError):
        binding.cs_packed_kv_append(new[:, :, :1].contiguous(), new[:, :, :1].contiguous(), pool, table, lens)
    with pytest.raises(TypeError):
        binding.cs_packed_kv_append(new.float(), new, pool, table, lens)
    with pytest.raises(binding.CacheSpecError):
        binding.cs_packed_kv_read(pool, table, lens, 0)
