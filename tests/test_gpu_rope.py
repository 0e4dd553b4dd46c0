"""Appends with the position rotation on the way, on the GPU, against the definition in
64 bits."""
import math

import numpy as np
import pytest
import torch

import ragged_reference as ref
import serving_reference as packed
from paper_2607_20507_gb300 import binding

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
EPS = 1e-6


def table_of_turns(n, rot, seed=0):
    angle = torch.arange(n, dtype=torch.float64)[:, None] * 10000.0 ** (-torch.arange(0, rot, 2, dtype=torch.float64) / rot)
    return torch.cat((angle.cos(), angle.sin()), 1).float().to(DEV)


def batch(ns, before, hq, hkv, ps, rot=128, seed=0, fused=True):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    T, B = sum(ns), len(ns)
    lens = torch.tensor([n + p for n, p in zip(ns, before)], dtype=torch.int32)
    cols = max(1, -(-int(lens.max()) // ps))
    P = B * cols + 2
    table = torch.randperm(P, generator=torch.Generator().manual_seed(seed))[:B * cols].reshape(B, cols).int()
    rows = torch.randn((T, hq + 2 * hkv, 128), generator=gen, device=DEV)
    rows = (rows * 2.0 ** torch.randint(-2, 3, (T, hq + 2 * hkv, 1), generator=gen, device=DEV)).bfloat16()
    qkv = [rows[:, :hq], rows[:, hq:hq + hkv], rows[:, hq + hkv:]]
    if not fused:
        qkv = [x.contiguous() for x in qkv]
    norms = [(1 + 0.3 * torch.randn(128, generator=gen, device=DEV)).bfloat16() for _ in range(2)]
    starts = torch.zeros(B + 1, dtype=torch.int32)
    starts[1:] = torch.tensor(ns).cumsum(0)
    return qkv, table_of_turns(cols * ps, rot), norms, table.to(DEV), lens.to(DEV), starts.to(DEV), P


def near(got, expect, before):
    """The rounding to bf16 (2^-8 of the value at most) and fp32 arithmetic: two products
    and a sum, after a norm (eight roundings of numbers of the row's size)."""
    bad = ~((got.double() - expect).abs() <= 1.01 * 2.0 ** -8 * expect.abs() + 2.0 ** -20 * before)
    assert not bad.any(), (int(bad.sum()), bad.nonzero()[:4].tolist(), got[bad][:4].tolist(), expect[bad][:4].tolist())


def expected(qkv, turns, norms, table, lens, starts, ps, P, positions, interleaved, eps):
    """(q_out rows, [(page, slot, key heads, value heads, row)]), 64 bits; None for a row left out."""
    q, k, v = [x.cpu() for x in qkv]
    turns = turns.cpu()
    norms = [None if n is None else n.cpu() for n in norms]
    table, T = table.cpu(), k.shape[0]
    out, kept = [None] * T, []
    for b, row, _, j in ref.rows_of(None if starts is None else starts.tolist(), lens.tolist(), table.shape[0], T,
                                    table.shape[1] * ps):
        t = j if positions is None else int(positions[row])
        if not 0 <= t < turns.shape[0]:
            continue
        out[row] = ref.turn(q[row], t, turns, norms[0], eps, interleaved)
        if j >= 0 and 0 <= int(table[b, j // ps]) < P:
            kept.append((int(table[b, j // ps]), j % ps, ref.turn(k[row], t, turns, norms[1], eps, interleaved), v[row], row))
    return out, kept


def check(ns, before, hq, hkv, ps, rot=128, norm=False, interleaved=False, fused=True, seed=0, positions=None, spoil=None,
          eps=EPS, starts_given=True, inplace=False):
    qkv, turns, norms, table, lens, starts, P = batch(ns, before, hq, hkv, ps, rot, seed, fused)
    norms = norms if norm else [None, None]
    if not starts_given:
        starts = None
    if spoil:
        table, lens = spoil(table, lens)
    pools = [torch.randn((P, hkv, ps, 128), device=DEV).bfloat16() for _ in range(2)]
    want = [p.clone() for p in pools]
    size = [p.clone().double() for p in pools]
    q_before = qkv[0].clone()
    out, kept = expected(qkv, turns, norms, table, lens, starts, ps, P, positions, interleaved, eps)
    given = qkv[0] if inplace else torch.full(qkv[0].shape, 9.0, dtype=torch.bfloat16, device=DEV)
    got = binding.cs_rope_kv_append(*qkv, turns, *pools, table, lens, starts, positions=positions, q_norm=norms[0],
                                    k_norm=norms[1], norm_eps=eps, interleaved=interleaved, q_out=given)
    assert got is given
    for row, x in enumerate(out):
        if x is None:
            assert torch.equal(got[row], q_before[row] if inplace else torch.full_like(got[row], 9.0))
        else:
            near(got[row].cpu(), x, x.abs().amax())
    k_want, v_want = want[0].double(), want[1]
    written = torch.zeros((P, ps), dtype=torch.bool, device=DEV)
    for page, slot, kx, vx, _ in kept:
        k_want[page, :, slot], v_want[page, :, slot], written[page, slot] = kx.to(DEV), vx.to(DEV), True
    assert torch.equal(pools[1], v_want)
    away = ~written
    assert torch.equal(pools[0].transpose(1, 2)[away], want[0].transpose(1, 2)[away])
    near(pools[0].transpose(1, 2)[written], k_want.transpose(1, 2)[written],
         k_want.transpose(1, 2)[written].abs().amax((-1, -2), keepdim=True))


@pytest.mark.parametrize("hq,hkv", [(8, 2), (1, 1), (7, 1), (28, 4), (64, 8), (5, 5), (36, 3)])
@pytest.mark.parametrize("norm", [False, True])
@pytest.mark.parametrize("interleaved", [False, True])
def test_heads(hq, hkv, norm, interleaved):
    check([1, 3, 0, 17], [5, 0, 9, 30], hq, hkv, 16, norm=norm, interleaved=interleaved, seed=hq)


@pytest.mark.parametrize("rot", [32, 64, 96, 128])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("fused", [False, True])
def test_dims_that_turn(rot, interleaved, fused):
    check([4, 1], [11, 200], 6, 2, 32, rot=rot, interleaved=interleaved, fused=fused, seed=rot)


@pytest.mark.parametrize("ps", [8, 16, 32, 64, 128, 256])
def test_pages(ps):
    check([1, 0, 0, 70, 2, 130], [0, 40, 0, ps - 1, 3 * ps, ps + 1], 4, 2, ps, norm=True, seed=ps)


def test_many_requests():
    check([(3 * b) % 4 for b in range(1300)], [b % 19 for b in range(1300)], 2, 1, 8)


@pytest.mark.parametrize("hq,hkv", [(128, 8), (63, 3), (12, 4)])
def test_heads_spread_over_warps(hq, hkv):
    check([300, 0, 1, 249], [3, 9, 100, 0], hq, hkv, 16, norm=True)


@pytest.mark.parametrize("inplace", [False, True])
@pytest.mark.parametrize("fused", [False, True])
def test_in_place(inplace, fused):
    check([9, 1, 4], [3, 70, 0], 8, 2, 16, norm=True, inplace=inplace, fused=fused)


def test_uniform_rows_need_no_starts():
    check([5] * 7, [b * 9 for b in range(7)], 8, 2, 16, starts_given=False)


def test_given_positions_and_those_outside_the_table():
    positions = torch.tensor([0, 3, 3, 63, 64, -1, 2 ** 30, 5, -2 ** 31, 9], dtype=torch.int32, device=DEV)
    check([6, 4], [50, 20], 8, 2, 16, positions=positions)


def test_pages_outside_the_pool_and_short_lengths():
    def spoil(table, lens):
        table[0, 0], table[1, 1], table[2, 0] = -1, 2 ** 30, -7
        return table, torch.tensor([5, 10 ** 6, 20], dtype=torch.int32, device=DEV)
    check([9, 20, 6], [10, 12, 14], 8, 2, 16, spoil=spoil)


def test_rows_of_nobody_stay():
    qkv, turns, norms, table, lens, starts, P = batch([2, 3], [5, 9], 4, 2, 16)
    pools = [torch.zeros((P, 2, 16, 128), dtype=torch.bfloat16, device=DEV) for _ in range(2)]
    expect = binding.cs_rope_kv_append(*qkv, turns, *pools, table, lens, starts)
    wide = [torch.nn.functional.pad(x, (0, 0, 0, 0, 3, 4), value=math.nan) for x in qkv]
    again = [torch.zeros_like(p) for p in pools]
    out = torch.full(wide[0].shape, 4.0, dtype=torch.bfloat16, device=DEV)
    binding.cs_rope_kv_append(*wide, turns, *again, table, lens, starts + 3, q_out=out)
    assert torch.equal(out[3:8], expect) and (out[:3] == 4.0).all() and (out[8:] == 4.0).all()
    assert all(torch.equal(a, b) for a, b in zip(pools, again))


def test_without_queries():
    qkv, turns, norms, table, lens, starts, P = batch([2, 30], [5, 9], 4, 2, 16)
    pools = [torch.zeros((P, 2, 16, 128), dtype=torch.bfloat16, device=DEV) for _ in range(2)]
    again = [torch.zeros_like(p) for p in pools]
    binding.cs_rope_kv_append(*qkv, turns, *pools, table, lens, starts)
    assert binding.cs_rope_kv_append(None, *qkv[1:], turns, *again, table, lens, starts) is None
    assert all(torch.equal(a, b) for a, b in zip(pools, again))


def test_no_turn_is_the_plain_append():
    qkv, turns, norms, table, lens, _, P = batch([6, 6, 6], [5, 9, 70], 4, 2, 16, fused=False)
    still = torch.cat((torch.ones_like(turns[:, :64]), torch.zeros_like(turns[:, 64:])), 1)
    pools = [torch.zeros((P, 2, 16, 128), dtype=torch.bfloat16, device=DEV) for _ in range(2)]
    again = [torch.zeros_like(p) for p in pools]
    out = binding.cs_rope_kv_append(*qkv, still, *pools, table, lens)
    binding.cs_kv_append(*(x.unflatten(0, (3, 6)) for x in qkv[1:]), *again, table, lens)
    assert torch.equal(out, qkv[0]) and all(torch.equal(a, b) for a, b in zip(pools, again))


def test_values_keep_their_bits_and_a_row_that_is_not_finite_is_its_own():
    qkv, turns, norms, table, lens, starts, P = batch([2, 30], [5, 9], 4, 2, 16)
    clean = [torch.zeros((P, 2, 16, 128), dtype=torch.bfloat16, device=DEV) for _ in range(2)]
    expect = binding.cs_rope_kv_append(*qkv, turns, *clean, table, lens, starts, q_norm=norms[0], k_norm=norms[1])
    qkv[0][1, 2], qkv[1][4, 1, 7] = math.nan, math.inf
    qkv[2][3, 0, :4] = torch.tensor([math.nan, -math.inf, -0.0, 1e-40], device=DEV)
    dirty = [torch.zeros_like(p) for p in clean]
    got = binding.cs_rope_kv_append(*qkv, turns, *dirty, table, lens, starts, q_norm=norms[0], k_norm=norms[1])
    same = (got == expect).all(-1)
    assert (~same).nonzero().tolist() == [[1, 2]]
    j = 9 + 4 - 2
    differ = (dirty[0].view(torch.int16) != clean[0].view(torch.int16)).any(-1).nonzero().tolist()
    assert differ == [[int(table[1, j // 16]), 1, j % 16]]
    row = dirty[1][int(table[1, (9 + 1) // 16]), 0, (9 + 1) % 16]
    assert torch.equal(row.view(torch.int16), qkv[2][3, 0].view(torch.int16))


# --------------------------------------------------------------- the packed cache
@pytest.mark.parametrize("rot", [32, 64, 96])
@pytest.mark.parametrize("interleaved", [False, True])
def test_dims_that_do_not_turn_stay_whatever_stands_beside_them(rot, interleaved):
    qkv, turns, _, table, lens, starts, P = batch([3, 30], [4, 0], 4, 2, 16, rot, seed=3)
    pools = [torch.zeros((P, 2, 16, 128), dtype=torch.bfloat16, device=DEV) for _ in range(2)]
    clean = binding.cs_rope_kv_append(*qkv, turns, *pools, table, lens, starts, interleaved=interleaved)
    clean_k = pools[0].clone()
    for x in qkv[:2]:
        x[1::2, :, rot::5], x[1::2, :, rot + 1::5], x[1::2, :, rot + 2::7], x[1::2, :, rot + 3::7] = math.inf, -0.0, -math.inf, 3e38
    got = binding.cs_rope_kv_append(*qkv, turns, *pools, table, lens, starts, interleaved=interleaved)
    assert torch.equal(got[..., :rot], clean[..., :rot]) and torch.equal(pools[0][..., :rot], clean_k[..., :rot])
    assert torch.equal(got[..., rot:].view(torch.int16), qkv[0][..., rot:].contiguous().view(torch.int16))
    for b, row, _, j in ref.rows_of(starts.tolist(), lens.tolist(), 2, 33, table.shape[1] * 16):
        put = pools[0][int(table[b, j // 16]), :, j % 16, rot:]
        assert torch.equal(put.view(torch.int16), qkv[1][row, :, rot:].contiguous().view(torch.int16))
    qkv[0][0, 0, rot + 9] = math.nan
    again = binding.cs_rope_kv_append(*qkv, turns, *pools, table, lens, starts, interleaved=interleaved)
    assert (again.isnan()).nonzero().tolist() == [[0, 0, rot + 9]]


def packed_pool(P, H, ps, heads, seed=0):
    rng = np.random.default_rng(seed)
    scales = [torch.from_numpy((2.0 ** rng.uniform(-3, 1, H)).astype(np.float32)).to(DEV) for _ in range(2)] if heads else [None] * 2
    pool = binding.packed_pool(P, H, ps, DEV, *scales)
    for t in pool[:4]:
        t.view(torch.uint8).fill_(0x5A)
    return pool


def host(t):
    return t.detach().cpu().view(torch.uint8).numpy() if t.dtype == torch.float8_e4m3fn else t.detach().cpu().numpy()


@pytest.mark.parametrize("ns,before,hq,hkv,ps,rot", [([1, 5, 0, 20], [0, 30, 4, 17], 8, 2, 16, 128), ([3], [2], 1, 1, 8, 64),
                                                     ([40, 1], [9, 300], 28, 4, 32, 96), ([2, 2, 2], [7, 8, 9], 5, 5, 64, 32),
                                                     ([70], [0], 6, 3, 128, 128)])
@pytest.mark.parametrize("heads", [False, True])
@pytest.mark.parametrize("interleaved", [False, True])
def test_packed(ns, before, hq, hkv, ps, rot, heads, interleaved):
    qkv, turns, norms, table, lens, starts, P = batch(ns, before, hq, hkv, ps, rot, seed=rot + hq)
    pool = packed_pool(P, hkv, ps, heads)
    out, kept = expected(qkv, turns, norms, table, lens, starts, ps, P, None, interleaved, EPS)
    got = binding.cs_packed_rope_kv_append(*qkv, turns, pool, table, lens, starts, q_norm=norms[0], k_norm=norms[1],
                                           norm_eps=EPS, interleaved=interleaved)
    plain = [torch.zeros((P, hkv, ps, 128), dtype=torch.bfloat16, device=DEV) for _ in range(2)]
    assert torch.equal(got, binding.cs_rope_kv_append(*qkv, turns, *plain, table, lens, starts, q_norm=norms[0],
                                                      k_norm=norms[1], norm_eps=EPS, interleaved=interleaved))
    kc, ks, vc, vs = (host(t) for t in pool[:4])
    kh, vh = (np.ones(hkv) if t is None else host(t).astype(np.float64) for t in pool[4:])
    left = np.ones((P, ps), bool)
    for page, slot, kx, vx, _ in kept:
        left[page, slot] = False
        codes, scales = packed.quantise(vx.float().numpy(), vh)
        assert np.array_equal(vc[page, :, slot], codes) and np.array_equal(vs[page, :, slot], scales)
        # keys: the code nearest to the 64-bit value, or one as near but for fp32's rounding
        x = kx.numpy()
        top = np.abs(x).reshape(hkv, 8, 16).max(-1)
        s = packed.e4m3_values()[ks[page, :, slot]]
        want = np.minimum(top / (6 * kh[:, None]), 448)
        best = packed.e4m3_values()[packed.to_e4m3(want)]
        assert (np.abs(s - want) <= np.abs(best - want) + 2.0 ** -18 * want).all()
        unit = (s * kh[:, None])[..., None]
        value = packed.values(kc[page, :, slot][:, None], ks[page, :, slot][:, None], kh)[:, 0].reshape(hkv, 8, 16)
        y = np.where(unit > 0, np.clip(x.reshape(hkv, 8, 16) / np.where(unit > 0, unit, 1), -6, 6), 0)
        code = np.where(unit > 0, value / np.where(unit > 0, unit, 1), 0)
        gap = np.abs(np.abs(y)[..., None] - packed.E2M1).min(-1)
        assert (np.abs(code - y) <= gap + 2.0 ** -17 * (np.abs(y) + np.abs(y).max(-1, keepdims=True))).all()
    assert (kc.transpose(0, 2, 1, 3)[left] == 0x5A).all() and (vs.transpose(0, 2, 1, 3)[left] == 0x5A).all()


def test_packed_values_that_are_not_finite():
    qkv, turns, _, table, lens, starts, P = batch([4], [3], 2, 2, 16)
    qkv[2][1, 0, 3], qkv[2][1, 1, 20], qkv[2][2, 0] = math.nan, math.inf, 0.0
    pool, plain = packed_pool(P, 2, 16, True), packed_pool(P, 2, 16, True)
    binding.cs_packed_rope_kv_append(*qkv, turns, pool, table, lens, starts)
    binding.cs_packed_kv_append(*(x.contiguous()[None] for x in qkv[1:]), plain, table, lens)
    assert torch.equal(pool.v_codes, plain.v_codes)
    assert torch.equal(pool.v_scales.view(torch.uint8), plain.v_scales.view(torch.uint8))


def test_captured_and_replayed():
    qkv, turns, norms, table, lens, starts, P = batch([3, 1, 9], [5, 40, 0], 8, 2, 16)
    pools = [torch.zeros((P, 2, 16, 128), dtype=torch.bfloat16, device=DEV) for _ in range(2)]
    out = torch.zeros((13, 8, 128), dtype=torch.bfloat16, device=DEV)
    call = lambda o, ps: binding.cs_rope_kv_append(*qkv, turns, *ps, table, lens, starts, q_norm=norms[0],  # noqa: E731
                                                   k_norm=norms[1], q_out=o)
    call(out, pools)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        call(out, pools)
    lens.copy_(torch.tensor([30, 33, 10]))
    starts.copy_(torch.tensor([0, 0, 6, 13]))
    out.zero_()
    for p in pools:
        p.zero_()
    graph.replay()
    again = [torch.zeros_like(p) for p in pools]
    assert torch.equal(out, call(None, again)) and all(torch.equal(a, b) for a, b in zip(pools, again))
