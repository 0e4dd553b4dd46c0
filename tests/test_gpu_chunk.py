"""Attention of every request's newest tokens over the paged cache, on the GPU, against
the definition in 64 bits."""
import math

import pytest
import torch

import ragged_reference as ref
from paper_2607_20507_gb300 import binding

pytestmark = pytest.mark.gpu

DEV = "cuda:0"


def batch(ns, before, hq, hkv, ps, seed=0, fused=False, spare=3, junk=True):
    """q, pools, table, lens and starts of requests with ns[b] new tokens after before[b]; slots of nobody hold NaN."""
    gen = torch.Generator(device=DEV).manual_seed(seed)
    T, B = sum(ns), len(ns)
    lens = torch.tensor([n + p for n, p in zip(ns, before)], dtype=torch.int32)
    need = [-(-int(L) // ps) for L in lens]
    cols = max(1, max(need))
    P = sum(need) + spare
    order = torch.randperm(P, generator=torch.Generator().manual_seed(seed + 1)).int()
    table = torch.full((B, cols), -1, dtype=torch.int32)
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = order[at:at + n]
        at += n
    pools = [torch.randn((P, hkv, ps, 128), generator=gen, device=DEV).bfloat16() for _ in range(2)]
    if junk:
        used = torch.zeros((P, ps), dtype=torch.bool)
        for b, L in enumerate(lens.tolist()):
            for j in range(L):
                used[table[b, j // ps], j % ps] = True
        for p in pools:
            p.transpose(1, 2)[~used.to(DEV)] = math.nan
    width = hq + 2 * hkv if fused else hq
    q = torch.randn((T, width, 128), generator=gen, device=DEV).bfloat16()[:, :hq]
    starts = torch.zeros(B + 1, dtype=torch.int32)
    starts[1:] = torch.tensor(ns).cumsum(0)
    return q, pools[0], pools[1], table.to(DEV), lens.to(DEV), starts.to(DEV)


def check(args, scale=None, **kw):
    q, k, v, table, lens, starts = args
    if scale is not None:
        kw["sm_scale"] = scale
    out = binding.cs_chunk_attention(q, k, v, table, lens, starts, **kw)
    expect, size = ref.attention(q, k, v, table, lens, starts, scale)
    # the output's rounding to bf16 and the weights' (8 significant bits: 2^-8 of the
    # value, or of every term, at most), and fp32 scores, exponents and sums
    tol = 1.01 * 2.0 ** -8 * expect.abs() + (1.01 * 2.0 ** -8 + 2.0 ** -13) * size + 1e-37
    bad = ~((out.double() - expect).abs() <= tol)
    assert not bad.any(), (int(bad.sum()), bad.nonzero()[:4].tolist(), out[bad][:4].tolist(), expect[bad][:4].tolist())
    return out


HEADS = [(8, 2), (7, 1), (4, 4), (64, 8), (5, 1), (32, 1), (71, 1), (128, 1), (9, 3)]


@pytest.mark.parametrize("hq,hkv", HEADS)
@pytest.mark.parametrize("n,before", [(1, 0), (1, 300), (3, 125), (37, 0), (130, 515)])
def test_one_request(hq, hkv, n, before):
    check(batch([n], [before], hq, hkv, 16, seed=n + hq))


@pytest.mark.parametrize("ps", [8, 16, 32, 64, 128, 256])
@pytest.mark.parametrize("seed", [0, 1])
def test_ragged(ps, seed):
    ns = [1, 70, 0, 1, 1, 33, 257, 2, 0, 5, 129, 64]
    before = [0, 300, 40, 1, 700, 1, 255, 126, 0, 127, 0, 1000]
    check(batch(ns, before, 8, 2, ps, seed, fused=bool(seed)))


@pytest.mark.parametrize("L", [1, 2, 15, 16, 17, 63, 64, 65, 127, 128, 129, 130, 255, 256, 257, 383, 385, 1023])
def test_lengths(L):
    check(batch([1, min(L, 31), L], [L - 1, L - min(L, 31), 0], 12, 3, 16, L))


@pytest.mark.parametrize("n", [1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 255, 256, 257, 300])
@pytest.mark.parametrize("G", [1, 3, 8])
def test_counts(n, G):
    check(batch([n, 1, n], [5, 77, 600], 2 * G, 2, 32, n))


def test_many_short_requests():
    ns = [(7 * b) % 5 for b in range(1500)]
    before = [(13 * b) % 90 for b in range(1500)]
    check(batch(ns, before, 4, 1, 16, junk=False))


def test_one_long_context_split_over_the_card():
    check(batch([1], [40000], 8, 1, 16, junk=False))
    check(batch([3, 1], [70001, 5], 2, 1, 64, junk=False))


def test_a_chunk_behind_a_long_context():
    check(batch([700], [9000], 16, 2, 16, junk=False))


@pytest.mark.parametrize("ns,before,hq,hkv", [
    ([1] * 100, [20] * 99 + [60000], 8, 2),                        # one context over many CTAs, among short ones
    ([1] * 90, [3000 + 37 * b for b in range(90)], 16, 2),
    ([300] * 12, [2000] * 12, 16, 4),                              # whole blocks of rows
    ([256, 1, 700] * 6, [100, 9000, 1500] * 6, 4, 4),
    ([3, 40] * 20, [6000 - 150 * b for b in range(40)], 28, 4),
])
def test_blocks_cut_between_ctas(ns, before, hq, hkv):
    """Whoever comes last joins the pieces of a block, in the same order."""
    args = batch(ns, before, hq, hkv, 16, junk=False)
    out = check(args)
    for _ in range(5):
        assert torch.equal(binding.cs_chunk_attention(*args), out)


@pytest.mark.parametrize("n", [1, 3, 70])
@pytest.mark.parametrize("L", [544, 639, 640, 641, 657, 720, 817, 832, 833, 960, 1100, 1301])
def test_few_blocks_of_lengths_that_are_just_cut(L, n):
    check(batch([n], [L - n], 8, 2, 16, seed=L + n, spare=0))


def test_one_context_of_many_pieces_beside_many_short_ones():
    ns = [1] * 40 + [2] + [1] * 39
    check(batch(ns, [63 + b for b in range(40)] + [20001] + [63] * 39, 4, 1, 64, seed=7))


def test_a_page_table_of_many_columns():
    """The schedule's weights in 64 bits, where a call's might not fit 32: the same results."""
    for ns, before in (([1, 300, 7, 0, 1, 64, 1, 2] * 2, [5000, 20, 900, 3, 1, 0, 16000, 300] * 2), ([300, 1], [9000, 20000])):
        q, k, v, table, lens, starts = batch(ns, before, 16, 2, 256, junk=False)
        out = check((q, k, v, table, lens, starts))
        wide = torch.full((len(ns), 1 << 22), -1, dtype=torch.int32, device=DEV)
        wide[:, :table.shape[1]] = table
        assert torch.equal(binding.cs_chunk_attention(q, k, v, wide, lens, starts), out)


def test_uniform_rows_need_no_starts():
    q, k, v, table, lens, starts = batch([4] * 6, [9, 0, 200, 33, 64, 1], 8, 2, 16)
    assert torch.equal(binding.cs_chunk_attention(q, k, v, table, lens), binding.cs_chunk_attention(q, k, v, table, lens, starts))


def test_rows_of_nobody_stay():
    q, k, v, table, lens, starts = batch([5, 0, 40], [9, 3, 200], 8, 2, 16)
    wide = torch.full((60, 8, 128), math.nan, device=DEV, dtype=torch.bfloat16)
    wide[7:52] = q
    out = torch.full_like(wide, 3.5)
    got = binding.cs_chunk_attention(wide, k, v, table, lens, starts + 7, out=out)
    assert got is out
    assert torch.equal(out[7:52], binding.cs_chunk_attention(q, k, v, table, lens, starts))
    assert (out[:7] == 3.5).all() and (out[52:] == 3.5).all()


def test_lengths_outside_what_a_row_holds_and_rows_without_keys():
    q, k, v, table, lens, starts = batch([6, 40, 3, 300], [0, 20, 10, 0], 8, 2, 16, junk=False)
    lens = torch.tensor([2, 100000, -5, 4], dtype=torch.int32, device=DEV)
    table = table.clamp(min=0)
    out = check((q, k, v, table, lens, starts))
    assert (out[:4] == 0).all() and (out[46:49] == 0).all() and (out[49:345] == 0).all()


def test_pages_outside_the_pool_read_as_zeros():
    q, k, v, table, lens, starts = batch([6, 140, 1], [50, 20, 300], 8, 2, 16, junk=False)
    table[0, 1], table[1, 0], table[1, 5], table[2, 7] = -1, k.shape[0], 2 ** 30, -2 ** 31
    check((q, k, v, table, lens, starts))


@pytest.mark.parametrize("scale", [0.01, 1.0, 4.0])
def test_scale(scale):
    q, k, v, table, lens, starts = batch([40, 1, 300], [50, 620, 0], 8, 2, 16)
    # (as the reference sees it: fp32)
    check((q, k, v, table, lens, starts), scale=float(torch.tensor(scale)))


def test_growing_scores_move_the_maximum():
    q, k, v, table, lens, starts = batch([300, 1], [300, 2000], 8, 2, 16, junk=False)
    q = (q.abs() / 8).contiguous()
    for b in range(2):
        for j in range(int(lens[b])):
            k[table[b, j // 16], :, j % 16] = k[table[b, j // 16], :, j % 16] / 64 + j / 64
    check((q, k, v, table, lens, starts))
    check((q, -k, v, table, lens, starts))


@pytest.mark.parametrize("big", [1e5, 3.3895e38])
def test_large_values(big):
    q, k, v, table, lens, starts = batch([70, 1], [300, 900], 8, 2, 16)
    v[table[0, 3].item(), :, 2] = big
    v[table[1, 20].item(), :, 5] = -big
    out = check((q, k, v, table, lens, starts))
    assert torch.isfinite(out).all()


def test_a_row_of_q_that_is_not_finite_is_its_own():
    q, k, v, table, lens, starts = batch([70, 1], [300, 900], 8, 2, 16)
    clean = binding.cs_chunk_attention(q, k, v, table, lens, starts)
    q[33, 5] = math.nan
    got = binding.cs_chunk_attention(q, k, v, table, lens, starts)
    keep = torch.ones(got.shape[:2], dtype=torch.bool, device=DEV)
    keep[33, 5] = False
    assert torch.equal(got[keep], clean[keep]) and torch.isnan(got[33, 5]).all()


def test_twice_is_the_same_and_the_status_is_clean():
    args = batch([300, 1, 77, 1], [500, 5000, 0, 31], 16, 2, 16)
    first = binding.cs_chunk_attention(*args)
    for _ in range(3):
        assert torch.equal(binding.cs_chunk_attention(*args), first)
    dims = binding.chunk_attn_dims(args[0], args[1], args[3])
    assert binding.cs_read_device_status(binding.chunk_attention_workspace(dims, args[0].shape[0], DEV)) == 0


def test_a_workspace_of_its_own_is_left_ready():
    """Zero-filled once; calls of other shapes in between find it as they need it."""
    args = batch([300, 1, 77, 1], [500, 5000, 0, 31], 16, 2, 16)
    other = batch([1] * 40 + [500], [3000] * 41, 8, 1, 32, junk=False)
    first, second = binding.cs_chunk_attention(*args), binding.cs_chunk_attention(*other)
    sizes = []
    for a in (args, other):
        dims = binding.chunk_attn_dims(a[0], a[1], a[3])
        sizes.append(binding.load_library().cs_chunk_attention_workspace_bytes(dims, a[0].shape[0]))
    ws = torch.zeros((max(sizes),), dtype=torch.uint8, device=DEV)
    for _ in range(3):
        assert torch.equal(binding.cs_chunk_attention(*args, workspace=ws), first)
        assert torch.equal(binding.cs_chunk_attention(*other, workspace=ws), second)
    assert binding.cs_read_device_status(ws) == 0


def test_captured_and_replayed_with_new_lengths():
    q, k, v, table, lens, starts = batch([300, 1, 77, 1], [500, 3000, 0, 31], 16, 2, 16, junk=False)
    table = table.clamp(min=0)
    out = torch.zeros((q.shape[0], 16, 128), dtype=torch.bfloat16, device=DEV)
    binding.cs_chunk_attention(q, k, v, table, lens, starts, out=out)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        binding.cs_chunk_attention(q, k, v, table, lens, starts, out=out)
    for new_lens, new_starts in (([800, 3001, 77, 32], [0, 300, 301, 378, 379]), ([64, 2222, 400, 32], [0, 3, 3, 299, 379])):
        lens.copy_(torch.tensor(new_lens))
        starts.copy_(torch.tensor(new_starts))
        out.fill_(7.0)
        graph.replay()
        assert torch.equal(out, binding.cs_chunk_attention(q, k, v, table, lens, starts))
        expect, size = ref.attention(q, k, v, table, lens, starts)
        assert ((out.double() - expect).abs() <= 1.01 * 2.0 ** -8 * (expect.abs() + size) + 2.0 ** -13 * size).all()


def test_on_streams_of_their_own():
    args = [batch([100, 1, 200], [600, 2000 + 100 * i, 3], 16, 2, 16, seed=i, junk=False) for i in range(3)]
    expect = [binding.cs_chunk_attention(*a) for a in args]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in args]
    for _ in range(5):
        got = []
        for s, a in zip(streams, args):
            with torch.cuda.stream(s):
                got.append(binding.cs_chunk_attention(*a))
        torch.cuda.synchronize()
        assert all(torch.equal(g, e) for g, e in zip(got, expect))


def test_it_agrees_with_verify_attention():
    q, k, v, table, lens, _ = batch([5] * 9, [60 * b for b in range(9)], 32, 8, 16)
    a = binding.cs_verify_attention(q.reshape(9, 5, 32, 128).contiguous(), k, v, table, lens, 4)
    b = binding.cs_chunk_attention(q, k, v, table, lens)
    _, size = ref.attention(q, k, v, table, lens, None)
    d = (a.double().flatten(0, 1) - b.double()).abs()
    assert (d <= 2.0 ** -7 * a.double().flatten(0, 1).abs() + (1.01 * 2.0 ** -8 + 2.0 ** -12) * size).all()


def test_nothing_to_do():
    q, k, v, table, lens, starts = batch([3], [20], 8, 2, 16)
    assert binding.cs_chunk_attention(q[:0], k, v, table, lens, starts * 0).shape == (0, 8, 128)
    assert binding.cs_chunk_attention(q[:0], k, v, table[:0], lens[:0]).shape == (0, 8, 128)
    out = torch.full((3, 8, 128), 2.0, dtype=torch.bfloat16, device=DEV)
    binding.cs_chunk_attention(q, k, v, table, lens, starts * 0, out=out)
    assert (out == 2.0).all()
