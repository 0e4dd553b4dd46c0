"""Rotated appends and chunk attention on the host: what they refuse before anything is enqueued, and their reference's
own pins.  No call here reaches a kernel."""
import ctypes
import math

import pytest
import torch

import ragged_reference as ref
from paper_2607_20507_gb300 import binding, build

FAKE = 0x10000
OK, BAD, UNSUPPORTED, NO_SPACE = binding.CS_OK, binding.CS_ERR_INVALID_ARG, binding.CS_ERR_UNSUPPORTED, binding.CS_ERR_WORKSPACE


@pytest.fixture(scope="module")
def lib():
    build.build()
    return binding.load_library()


def dims(**kw):
    d = dict(batch=4, n_q_heads=32, n_kv_heads=8, head_dim=128, page_size=16, max_pages_per_seq=64, num_pages=256,
             sm_scale=0.0)
    d.update(kw)
    return ctypes.byref(binding.AttnDims(*d.values()))


def turns(**kw):
    d = dict(tokens=8, rot_dim=128, interleaved=0, n_positions=1024, norm_eps=1e-6, q_stride=4096, k_stride=1024,
             v_stride=1024, q_out_stride=4096)
    d.update(kw)
    return ctypes.byref(binding.RopeDims(*d.values()))


def pool(**kw):
    d = dict(k_codes=FAKE, k_scales=FAKE, v_codes=FAKE, v_scales=FAKE, k_head_scale=None, v_head_scale=None)
    d.update(kw)
    return ctypes.byref(binding.PackedPoolPtrs(*d.values()))


def attend(lib, d=None, q=FAKE, stride=4096, tokens=8, k=FAKE, v=FAKE, table=FAKE, lens=FAKE, starts=FAKE, out=FAKE, ws=FAKE,
           n=1 << 40):
    return lib.cs_chunk_attention(d or dims(), q, stride, tokens, k, v, table, lens, starts, out, ws, n, None)


def append(lib, d=None, r=None, q=FAKE, k=FAKE, v=FAKE, cos=FAKE, pos=None, qn=None, kn=None, qo=FAKE, kp=FAKE, vp=FAKE,
           table=FAKE, lens=FAKE, starts=FAKE):
    return lib.cs_rope_kv_append(d or dims(), r or turns(), q, k, v, cos, pos, qn, kn, qo, kp, vp, table, lens, starts, None)


def packed(lib, d=None, r=None, q=FAKE, k=FAKE, v=FAKE, cos=FAKE, pos=None, qn=None, kn=None, qo=FAKE, p=None, table=FAKE,
           lens=FAKE, starts=FAKE):
    return lib.cs_packed_rope_kv_append(d or dims(), r or turns(), q, k, v, cos, pos, qn, kn, qo, p or pool(), table, lens,
                                        starts, None)


GEOMETRY = [(dict(batch=-1), BAD), (dict(n_q_heads=0), BAD), (dict(n_q_heads=30), BAD), (dict(n_kv_heads=0), BAD),
            (dict(head_dim=64), UNSUPPORTED), (dict(page_size=12), UNSUPPORTED), (dict(page_size=0), BAD),
            (dict(max_pages_per_seq=0), BAD), (dict(max_pages_per_seq=1 << 27), BAD), (dict(num_pages=0), BAD),
            (dict(sm_scale=float("nan")), BAD), (dict(sm_scale=float("inf")), BAD),
            (dict(num_pages=1 << 30, n_kv_heads=8), UNSUPPORTED)]


@pytest.mark.parametrize("kw,code", GEOMETRY + [(dict(n_q_heads=129, n_kv_heads=1), UNSUPPORTED)])
def test_attention_refuses_dims(lib, kw, code):
    assert attend(lib, dims(**kw), stride=1 << 20) == code
    assert lib.cs_last_error()
    assert lib.cs_chunk_attention_workspace_bytes(dims(**kw), 8) == 0


def test_attention_refuses_arguments(lib):
    assert attend(lib, tokens=-1) == BAD and attend(lib, tokens=1 << 27) == UNSUPPORTED
    assert [attend(lib, stride=s) for s in (0, 4088, 4100, -4096, 1 << 40)] == [BAD] * 5
    for name in ("q", "k", "v", "table", "lens", "out"):
        assert attend(lib, **{name: None}) == BAD
    for name in ("q", "k", "v", "out"):
        assert attend(lib, **{name: FAKE + 8}) == BAD
    for name in ("table", "lens", "starts"):
        assert attend(lib, **{name: FAKE + 2}) == BAD
    assert attend(lib, starts=None, tokens=7) == BAD
    assert attend(lib, ws=None) == NO_SPACE and attend(lib, n=16) == NO_SPACE and attend(lib, ws=FAKE + 16) == BAD
    assert lib.cs_chunk_attention(None, FAKE, 4096, 8, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, 1 << 40, None) == BAD
    assert attend(lib, dims(batch=0), q=None, out=None, ws=None) == OK and attend(lib, tokens=0, q=None, ws=None) == OK
    assert lib.cs_chunk_attention_workspace_bytes(dims(), -1) == 0


@pytest.mark.parametrize("call", [append, packed])
@pytest.mark.parametrize("kw,code", GEOMETRY)
def test_append_refuses_dims(lib, call, kw, code):
    assert call(lib, dims(**kw), turns(q_stride=1 << 20, q_out_stride=1 << 20)) == code
    assert lib.cs_last_error()


@pytest.mark.parametrize("call", [append, packed])
def test_append_refuses_arguments(lib, call):
    for kw, code in ((dict(tokens=-1), BAD), (dict(rot_dim=0), UNSUPPORTED), (dict(rot_dim=48), UNSUPPORTED),
                     (dict(rot_dim=160), UNSUPPORTED), (dict(interleaved=2), BAD), (dict(n_positions=0), BAD),
                     (dict(norm_eps=-1.0), BAD), (dict(norm_eps=math.nan), BAD), (dict(norm_eps=math.inf), BAD),
                     (dict(q_stride=4088), BAD), (dict(k_stride=1020), BAD), (dict(v_stride=1028), BAD),
                     (dict(q_out_stride=0), BAD)):
        assert call(lib, r=turns(**kw)) == code, kw
    for name in ("k", "v", "cos", "table", "lens", "q", "qo"):
        assert call(lib, **{name: None}) == BAD, name
    for name in ("q", "k", "v", "cos", "qn", "kn", "qo"):
        assert call(lib, **{name: FAKE + 8}) == BAD, name
    for name in ("pos", "table", "lens", "starts"):
        assert call(lib, **{name: FAKE + 2}) == BAD, name
    assert call(lib, r=turns(tokens=7), starts=None) == BAD
    assert call(lib, dims(batch=0), k=None) == OK and call(lib, r=turns(tokens=0), k=None) == OK


@pytest.mark.parametrize("call", [append, packed])
def test_append_refuses_queries_in_place_with_another_stride(lib, call):
    assert call(lib, r=turns(q_stride=8192)) == BAD and call(lib, r=turns(q_out_stride=4104)) == BAD


def test_append_refuses_pools(lib):
    assert append(lib, kp=None) == BAD and append(lib, vp=FAKE + 8) == BAD
    for name in ("k_codes", "k_scales", "v_codes", "v_scales"):
        assert packed(lib, p=pool(**{name: None})) == BAD and packed(lib, p=pool(**{name: FAKE + 8})) == BAD
    assert packed(lib, p=pool(v_head_scale=FAKE + 2)) == BAD
    for call, more in ((lib.cs_rope_kv_append, (FAKE, FAKE)), (lib.cs_packed_rope_kv_append, (pool(),))):
        args = (FAKE, FAKE, FAKE, FAKE, None, None, None, FAKE) + more + (FAKE, FAKE, FAKE, None)
        assert call(None, turns(), *args) == BAD and call(dims(), None, *args) == BAD
    assert lib.cs_packed_rope_kv_append(dims(), turns(), FAKE, FAKE, FAKE, FAKE, None, None, None, FAKE, None, FAKE, FAKE,
                                        FAKE, None) == BAD


def test_binding_refuses_tensors_of_the_host():
    x = torch.zeros((4, 2, 128), dtype=torch.bfloat16)
    pages = torch.zeros((3, 2, 16, 128), dtype=torch.bfloat16)
    ints = torch.zeros((1, 3), dtype=torch.int32)
    with pytest.raises(ValueError):
        binding.cs_chunk_attention(x, pages, pages, ints, ints[0, :1])
    with pytest.raises(TypeError):
        binding.cs_chunk_attention(x.float(), pages, pages, ints, ints[0, :1])
    with pytest.raises(ValueError):
        binding.cs_rope_kv_append(x, x, x, torch.zeros((48, 128)), pages, pages, ints, ints[0, :1])
    with pytest.raises(ValueError):
        binding.cs_packed_rope_kv_append(x, x, x, torch.zeros((48, 128)), binding.packed_pool(3, 2, 16, "cpu"), ints,
                                         ints[0, :1])


# ------------------------------------------------------------------ the reference
def test_reference_attention_is_dense_attention():
    gen = torch.Generator().manual_seed(3)
    ns, before, ps = [3, 0, 1, 6], [5, 2, 0, 9], 4
    T, B = sum(ns), len(ns)
    q = torch.randn((T, 6, 128), generator=gen)
    lens = torch.tensor([n + p for n, p in zip(ns, before)])
    dense = [torch.randn((B, 2, 15, 128), generator=gen) for _ in range(2)]
    table = torch.randperm(20, generator=gen)[:16].reshape(4, 4)
    pools = [torch.zeros((20, 2, ps, 128)) for _ in range(2)]
    for b in range(B):
        for j in range(15):
            for p, x in zip(pools, dense):
                p[table[b, j // ps], :, j % ps] = x[b, :, j]
    starts = torch.tensor([0] + ns).cumsum(0)
    out, size = ref.attention(q, *pools, table, lens, starts)
    at = 0
    for b, n in enumerate(ns):
        for i in range(n):
            L = before[b] + i + 1
            k, v = (x[b, :, :L].double().repeat_interleave(3, 0) for x in dense)
            p = torch.softmax(torch.einsum("hd,hld->hl", q[at].double(), k) / math.sqrt(128), -1)
            assert torch.allclose(out[at], torch.einsum("hl,hld->hd", p, v), atol=1e-12)
            assert (size[at] >= out[at].abs() - 1e-12).all()
            at += 1


def test_reference_turn_is_a_rotation():
    gen = torch.Generator().manual_seed(3)
    x = torch.randn((4, 128), generator=gen).double()
    for rot in (32, 128):
        angle = torch.rand((5, rot // 2), generator=gen).double() * 6
        table = torch.cat((angle.cos(), angle.sin()), 1)
        for interleaved in (False, True):
            y = ref.turn(x, 3, table, None, 0.0, interleaved)
            a, b = (slice(0, rot, 2), slice(1, rot, 2)) if interleaved else (slice(0, rot // 2), slice(rot // 2, rot))
            z = torch.complex(x[:, a], x[:, b]) * torch.exp(1j * angle[3])
            assert torch.allclose(y[:, a], z.real) and torch.allclose(y[:, b], z.imag)
            assert torch.equal(y[:, rot:], x[:, rot:])
    norm = torch.full((128,), 2.0)
    y = ref.turn(x, 3, table, norm, 0.0, False)
    assert torch.allclose(y.square().mean(-1), torch.full((4,), 4.0).double())


def test_reference_rows():
    assert list(ref.rows_of([1, 3, 3, 4], [7, 5, 2], 3, 6, 6)) == [(0, 1, 0, 4), (0, 2, 1, 5), (2, 3, 0, 1)]
    assert [r[:2] for r in ref.rows_of(None, [7, 5], 2, 4, 6)] == [(0, 0), (0, 1), (1, 2), (1, 3)]
