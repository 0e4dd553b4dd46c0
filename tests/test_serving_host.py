"""The packed cache, page and log-probability calls on the host: what they refuse before anything is enqueued,
and the references' own pins.  No call here reaches a kernel."""
import ctypes

import numpy as np
import pytest

import serving_reference as ref
from paper_2607_20507_gb300 import binding, build

FAKE = 0x10000
BAD, UNSUPPORTED, NO_SPACE = binding.CS_ERR_INVALID_ARG, binding.CS_ERR_UNSUPPORTED, binding.CS_ERR_WORKSPACE


@pytest.fixture(scope="module")
def lib():
    build.build()
    return binding.load_library()


def dims(**kw):
    d = dict(batch=4, n_q_heads=32, n_kv_heads=8, head_dim=128, page_size=16, max_pages_per_seq=64, num_pages=256,
             sm_scale=0.0)
    d.update(kw)
    return ctypes.byref(binding.AttnDims(*d.values()))


def pool(**kw):
    d = dict(k_codes=FAKE, k_scales=FAKE, v_codes=FAKE, v_scales=FAKE, k_head_scale=None, v_head_scale=None)
    d.update(kw)
    return ctypes.byref(binding.PackedPoolPtrs(*d.values()))


def attend(lib, d=None, p=None, k=4, q=FAKE, table=FAKE, lens=FAKE, out=FAKE, ws=FAKE, n=1 << 40):
    return lib.cs_packed_verify_attention(d or dims(), q, p or pool(), table, lens, k, out, ws, n, None)


@pytest.mark.parametrize("kw,code", [
    (dict(batch=-1), BAD), (dict(n_q_heads=0), BAD), (dict(n_q_heads=30), BAD), (dict(n_kv_heads=0), BAD),
    (dict(head_dim=64), UNSUPPORTED), (dict(page_size=12), UNSUPPORTED), (dict(page_size=0), BAD),
    (dict(max_pages_per_seq=0), BAD), (dict(max_pages_per_seq=1 << 27), BAD), (dict(num_pages=0), BAD),
    (dict(sm_scale=float("nan")), BAD), (dict(sm_scale=float("inf")), BAD),
    (dict(n_q_heads=512), UNSUPPORTED),     # 5 * 64 query rows
])
def test_attention_refuses_dims(lib, kw, code):
    assert attend(lib, dims(**kw)) == code
    assert lib.cs_last_error()
    assert lib.cs_packed_verify_attention_workspace_bytes(dims(**kw), 4) == 0


def test_attention_refuses_arguments(lib):
    assert [attend(lib, k=k) for k in (-1, 17)] == [BAD, BAD]
    for name in ("k_codes", "k_scales", "v_codes", "v_scales"):
        assert attend(lib, p=pool(**{name: None})) == BAD
        assert attend(lib, p=pool(**{name: FAKE + 8})) == BAD
    assert attend(lib, p=pool(k_head_scale=FAKE + 2)) == BAD
    for name in ("q", "table", "lens", "out"):
        assert attend(lib, **{name: None}) == BAD
    assert attend(lib, q=FAKE + 2) == BAD and attend(lib, out=FAKE + 4) == BAD and attend(lib, lens=FAKE + 1) == BAD
    assert attend(lib, ws=None) == NO_SPACE and attend(lib, n=16) == NO_SPACE and attend(lib, ws=FAKE + 16) == BAD
    assert lib.cs_packed_verify_attention(dims(), FAKE, None, FAKE, FAKE, 4, FAKE, FAKE, 1 << 40, None) == BAD
    assert lib.cs_packed_verify_attention(None, FAKE, pool(), FAKE, FAKE, 4, FAKE, FAKE, 1 << 40, None) == BAD
    assert attend(lib, dims(batch=0), q=None, out=None, ws=None) == binding.CS_OK


def test_rows_refuse(lib):
    def append(d=None, p=None, k=FAKE, v=FAKE, table=FAKE, lens=FAKE, n=5):
        return lib.cs_packed_kv_append(d or dims(), p or pool(), k, v, table, lens, n, None)

    def read(d=None, p=None, k=FAKE, v=FAKE, table=FAKE, lens=FAKE, n=5):
        return lib.cs_packed_kv_read(d or dims(), p or pool(), table, lens, n, k, v, None)

    for call in (append, read):
        assert call(n=0) == BAD and call(n=-3) == BAD
        for name in ("k", "v", "table", "lens"):
            assert call(**{name: None}) == BAD
        assert call(k=FAKE + 2) == BAD and call(v=FAKE + 8) == BAD and call(table=FAKE + 2) == BAD
        assert call(d=dims(head_dim=96)) == UNSUPPORTED and call(d=dims(page_size=24)) == UNSUPPORTED
        assert call(d=dims(n_kv_heads=-1)) == BAD and call(d=dims(batch=-2)) == BAD
        assert call(p=pool(v_scales=None)) == BAD and call(p=pool(k_scales=FAKE + 8)) == BAD
        assert call(d=dims(batch=0), k=None) == binding.CS_OK
    assert append(n=4097) == BAD


def page_dims(**kw):
    d = dict(rows=4, max_pages_per_seq=8, page_size=16, num_pages=100)
    d.update(kw)
    return ctypes.byref(binding.PageDims(*d.values()))


def pools(*entries):
    return (binding.PagePool * max(len(entries), 1))(*entries)


def test_pages_refuse(lib):
    one = pools((FAKE, 64))

    def fork(d=None, p=one, np_=1, table=FAKE, lens=FAKE, refs=FAKE, src=FAKE, dst=FAKE, n=2, room=0, out=FAKE, ws=FAKE,
             size=1 << 40):
        return lib.cs_kv_fork(d or page_dims(), p, np_, table, lens, refs, src, dst, n, room, out, ws, size, None)

    def compact(d=None, p=one, np_=1, table=FAKE, refs=FAKE, out=FAKE, ws=FAKE, size=1 << 40):
        return lib.cs_kv_compact(d or page_dims(), p, np_, table, refs, out, ws, size, None)

    def release(d=None, table=FAKE, lens=FAKE, refs=FAKE, rows=FAKE, keep=FAKE, n=2):
        return lib.cs_kv_release(d or page_dims(), table, lens, refs, rows, keep, n, None)

    for call in (fork, compact, release):
        for name in ("rows", "max_pages_per_seq", "page_size", "num_pages"):
            assert call(page_dims(**{name: 0})) == BAD
        assert call(page_dims(max_pages_per_seq=1 << 27)) == BAD
        assert call(table=None) == BAD and call(refs=None) == BAD and call(refs=FAKE + 2) == BAD
    for call in (fork, compact):
        assert call(np_=-1) == BAD and call(np_=129) == BAD and call(p=None) == BAD
        assert call(p=pools((None, 64))) == BAD and call(p=pools((FAKE + 8, 64))) == BAD
        assert call(p=pools((FAKE, 0))) == BAD and call(p=pools((FAKE, 24))) == BAD
        assert call(ws=None) == NO_SPACE and call(size=8) == NO_SPACE and call(ws=FAKE + 128) == BAD and call(out=None) == BAD
    assert fork(n=-1) == BAD and fork(room=-1) == BAD and fork(src=None) == BAD and fork(dst=FAKE + 1) == BAD
    assert release(n=-1) == BAD and release(rows=None) == BAD and release(keep=FAKE + 3) == BAD
    assert fork(n=0, src=None) == binding.CS_OK and release(n=0, rows=None) == binding.CS_OK
    assert lib.cs_kv_fork_workspace_bytes(page_dims(), -1) == 0
    assert lib.cs_kv_compact_workspace_bytes(page_dims(num_pages=0)) == 0


def test_logprobs_refuse(lib):
    def call(T=1.0, z=FAKE, tok=FAKE, lp=FAKE, ent=FAKE, ids=FAKE, top=FAKE, **kw):
        d = dict(rows=4, vocab=1000, logit_dtype=binding.CS_F32, n_top=5, row_stride=1000)
        d.update(kw)
        return lib.cs_logprobs(ctypes.byref(binding.LogprobDims(*d.values())), z, tok, T, lp, ent, ids, top, None)

    assert lib.cs_logprobs(None, FAKE, FAKE, 1.0, FAKE, FAKE, FAKE, FAKE, None) == BAD
    assert call(rows=-1) == BAD and call(vocab=0) == BAD and call(logit_dtype=2) == BAD
    assert call(n_top=-1) == BAD and call(n_top=33) == BAD and call(row_stride=999) == BAD
    assert call(row_stride=1 << 60) == BAD and call(vocab=(1 << 22) + 1, row_stride=1 << 23) == UNSUPPORTED
    assert [call(T=T) for T in (0.0, -1.0, float("inf"), float("nan"))] == [BAD] * 4
    assert call(z=None) == BAD and call(tok=None) == BAD and call(lp=None) == BAD and call(ids=None) == BAD
    assert call(z=FAKE + 2) == BAD and call(tok=FAKE + 1) == BAD and call(ent=FAKE + 2) == BAD
    assert call(rows=0, z=None) == binding.CS_OK


# ------------------------------------------------------- pins of the references
def test_reference_e4m3():
    torch = pytest.importorskip("torch")
    b = np.arange(256, dtype=np.uint8)
    np.testing.assert_array_equal(ref.e4m3_values(), torch.from_numpy(b).view(torch.float8_e4m3fn).double().numpy())
    x = np.concatenate((np.linspace(0, 448, 40001), 2.0 ** np.linspace(-12, 8.8, 5000))).astype(np.float32)
    expect = torch.from_numpy(x).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    np.testing.assert_array_equal(ref.to_e4m3(x), expect)


def test_reference_quantise():
    """A row on the grid is kept; any other is off by half a step at most."""
    grid = np.tile(np.concatenate((ref.E2M1, -ref.E2M1)), 8)[None, None] * 0.75
    c, s = ref.quantise(grid, np.ones(1))
    np.testing.assert_array_equal(ref.values(c.swapaxes(0, 1), s.swapaxes(0, 1), np.ones(1))[0], grid[0])
    x = np.random.default_rng(0).standard_normal((50, 3, 128)).astype(np.float32)
    head = np.array([1.0, 0.3, 2.7], np.float32)
    c, s = ref.quantise(x, head)
    v = ref.values(c.swapaxes(0, 1), s.swapaxes(0, 1), head).swapaxes(0, 1)
    top = np.abs(x).reshape(50, 3, 8, 16).max(-1).repeat(16, -1)
    assert (np.abs(v - x) <= top * (1 / 6 + 1 / 16)).all()


def test_reference_attention_and_logprobs():
    torch = pytest.importorskip("torch")
    rng = np.random.default_rng(1)
    k, v = rng.standard_normal((2, 4, 2, 8, 128))
    q = rng.standard_normal((1, 3, 4, 128))
    out, _ = ref.packed_attention(q, k, v, np.array([[2, 0, 3]], np.int32), np.array([21]), 0.1)
    rows = [np.concatenate([x[p] for p in (2, 0, 3)], 1)[:, :21] for x in (k, v)]
    seen = torch.ones(3, 21, dtype=torch.bool).tril(18)
    e = torch.nn.functional.scaled_dot_product_attention(
        torch.from_numpy(q[0]).permute(1, 0, 2), *(torch.from_numpy(r).repeat_interleave(2, 0) for r in rows), attn_mask=seen,
        scale=0.1)
    np.testing.assert_allclose(out[0], e.permute(1, 0, 2).numpy(), rtol=1e-10, atol=1e-12)
    z = rng.standard_normal((4, 50))
    lp, ent, ids, top = ref.logprobs(z, np.array([3, 0, 49, -1]), 0.7, 5)
    full = torch.log_softmax(torch.from_numpy(z) / 0.7, 1)
    np.testing.assert_allclose(lp[:3], [full[0, 3], full[1, 0], full[2, 49]], rtol=1e-12)
    np.testing.assert_allclose(ent[:3], torch.distributions.Categorical(logits=full[:3]).entropy().numpy(), rtol=1e-12)
    np.testing.assert_allclose(top[:3], torch.topk(full[:3], 5).values.numpy(), rtol=1e-12)
    assert lp[3] == -np.inf and (ids[3] == -1).all()
