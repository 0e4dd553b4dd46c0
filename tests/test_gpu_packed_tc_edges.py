"""Packed attention at the edges with more than 24 query rows a KV head: the tcgen05 form's columns of 32, 48, 64 and 80
and its row blocks.  Against the definition in 64 bits."""
import numpy as np
import pytest
import torch

from paper_2607_20507_gb300 import binding
from test_gpu_packed import DEV, check_attention, dense, random_pool, table_of

pytestmark = pytest.mark.gpu

# (rows of a request, query heads a KV head): 28, 35, 56, 72 and 80 rows a span, 136 in two blocks, 85 in two uneven ones
FORMS = [(4, 7), (5, 7), (7, 8), (9, 8), (10, 8), (17, 8), (17, 5)]


def queries(B, rows, Hq, seed, size=1.0):
    return (torch.randn(B, rows, Hq, 128, generator=torch.Generator().manual_seed(seed)) * size).bfloat16().to(DEV)


@pytest.mark.parametrize("rows,G", FORMS)
def test_many_ragged_requests(rows, G):
    """More requests than a launch schedules at a time, most of them short."""
    rng = np.random.default_rng(rows * G)
    B, ps, cols, P = 1100, 16, 10, 400
    lens = np.minimum(rng.geometric(0.02, B), cols * ps).astype(np.int32)
    lens[rng.integers(0, B, 40)] = 0
    table = rng.integers(0, P, (B, cols)).astype(np.int32)   # (pages shared by several rows)
    check_attention(queries(B, rows, G, 1), random_pool(rng, P, 1, ps), table, lens, rows - 1)


@pytest.mark.parametrize("rows,G", [(5, 7), (9, 8), (17, 8)])
def test_pool_past_32_bits(rows, G):
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
    q = queries(2, rows, H * G, 9)
    want = check_attention(q, small, np.arange(4, dtype=np.int32).reshape(2, 2), lens, rows - 1)
    got = binding.cs_packed_verify_attention(q, big, torch.from_numpy(at).to(DEV), torch.from_numpy(lens).to(DEV), rows - 1)
    assert torch.equal(got, want)


@pytest.mark.parametrize("rows,G", FORMS)
def test_pages_outside_the_pool_read_as_zeros(rows, G):
    rng = np.random.default_rng(12)
    B, ps, cols, P = 4, 16, 20, 80
    pool = random_pool(rng, P, 2, ps)
    table = table_of(rng, B, cols, P)
    table[1, 2], table[1, 9], table[2] = P, -1, np.resize((-1, -5, 1 << 30, P, P + 1, -(1 << 31)), cols)
    out = check_attention(queries(B, rows, 2 * G, 3), pool, table, np.array([320, 317, 250, 1 << 30], np.int32), rows - 1)
    assert (out[2] == 0).all()


@pytest.mark.parametrize("rows,G", FORMS)
def test_never_sees_slots_past_the_context(rows, G):
    """Every byte past L, NaN scales among them, and the pages past the last one; rows that see no key at all."""
    rng = np.random.default_rng(13)
    ps, cols, H = 32, 9, 2
    lens = np.array([1, rows - 1, rows, 31, 33, 127, 128, 129, 255, 257], np.int32)
    B = len(lens)
    P = B * cols
    pool = random_pool(rng, P, H, ps)
    table = table_of(rng, B, cols, P)
    kv = dense(pool)
    for b in range(B):
        for pos in range(lens[b], cols * ps):
            for t in pool[:4]:
                t.view(torch.uint8)[table[b, pos // ps], :, pos % ps] = 0x7F
        table[b, -(-int(lens[b]) // ps):] = 1 << 29
    out = check_attention(queries(B, rows, H * G, 4), pool, table, lens, rows - 1, kv=kv)
    assert (out[0, :rows - 1] == 0).all()


@pytest.mark.parametrize("rows,G", FORMS)
@pytest.mark.parametrize("size", [1e-30, 1e-6, 300.0, 3e4])
def test_query_sizes(rows, G, size):
    """Queries far from 1: fp16 would lose the first two and overflow at the last."""
    rng = np.random.default_rng(14)
    pool = random_pool(rng, 24, 2, 16, heads=False)
    check_attention(queries(2, rows, 2 * G, 5, size), pool, table_of(rng, 2, 12, 24), np.array([190, 129], np.int32), rows - 1,
                    sm_scale=0.05 / size)


@pytest.mark.parametrize("rows,G", FORMS)
def test_one_key_outweighs_the_rest(rows, G):
    """A score hundreds above the others, early, late and in the middle of the context."""
    rng = np.random.default_rng(15)
    ps, cols, H = 16, 40, 1
    pool = random_pool(rng, 3 * cols, H, ps, heads=False)
    table = table_of(rng, 3, cols, 3 * cols)
    for b, pos in enumerate((0, 333, 620)):
        pool.k_codes[table[b, pos // ps], :, pos % ps] = 0x77
        pool.k_scales.view(torch.uint8)[table[b, pos // ps], :, pos % ps] = 0x58
    q = torch.rand(3, rows, G, 128, generator=torch.Generator().manual_seed(6)).bfloat16().to(DEV)
    check_attention(q, pool, table, np.array([640, 640, 640], np.int32), rows - 1)


@pytest.mark.parametrize("rows,G", [(1, 4), (3, 7)] + FORMS)
@pytest.mark.parametrize("above", [14.0, 22.0, 45.0, 80.0])
def test_outputs_that_rest_on_faint_weights(rows, G, above):
    """One key some tens of nats above the others, whose value is 0: the output is what the others leave."""
    rng = np.random.default_rng(18)
    ps, cols, H, L = 16, 20, 1, 300
    pool = random_pool(rng, 2 * cols, H, ps, heads=False)
    table = table_of(rng, 2, cols, 2 * cols)
    pool.k_codes[..., :8] = 0                                       # the first group: 0 but for the one key
    for b, pos in enumerate((3, 200)):
        page, slot = table[b, pos // ps], pos % ps
        pool.k_codes[page, :, slot, :8], pool.v_codes[page, :, slot] = 0x77, 0
        pool.k_scales.view(torch.uint8)[page, :, slot, 0] = 0x38    # 16 dims of 6 times 1
    q = queries(2, rows, G, 19, 0.05)
    q[..., :16] = above / 96
    check_attention(q, pool, table, np.array([L, L], np.int32), rows - 1, sm_scale=1.0)


@pytest.mark.parametrize("rows,G", FORMS)
def test_query_at_any_address(rows, G):
    rng = np.random.default_rng(17)
    pool = random_pool(rng, 24, 2, 16)
    table = table_of(rng, 2, 12, 24)
    flat = torch.randn(2 * rows * 2 * G * 128 + 2, generator=torch.Generator().manual_seed(8)).bfloat16().to(DEV)
    q = flat[2:].view(2, rows, 2 * G, 128)
    assert q.data_ptr() % 16 == 4
    check_attention(q, pool, table, np.array([190, 33], np.int32), rows - 1)


@pytest.mark.parametrize("rows,G", [(1, 4), (3, 7)] + FORMS)
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_a_query_that_is_no_number_stays_with_its_row(rows, G, bad):
    rng = np.random.default_rng(20)
    B, ps, cols, H = 2, 16, 30, 2
    pool = random_pool(rng, B * cols, H, ps)
    table = torch.from_numpy(table_of(rng, B, cols, B * cols)).to(DEV)
    lens = torch.tensor([470, 200], dtype=torch.int32, device=DEV)
    q = queries(B, rows, H * G, 21)
    want = binding.cs_packed_verify_attention(q, pool, table, lens, rows - 1)
    spoilt = q.clone()
    spoilt[1, rows - 1, G, 5] = bad
    got = binding.cs_packed_verify_attention(spoilt, pool, table, lens, rows - 1)
    assert torch.isnan(got[1, rows - 1, G]).any()
    got[1, rows - 1, G] = want[1, rows - 1, G]
    # (a tile that takes the longer way for one row does so for all: the last bits may differ)
    torch.testing.assert_close(got.float(), want.float(), rtol=2.0 ** -7, atol=2.0 ** -9)


@pytest.mark.parametrize("rows,G", FORMS)
def test_same_bits_every_time(rows, G):
    rng = np.random.default_rng(16)
    B, ps, cols, H = 9, 16, 60, 4
    pool = random_pool(rng, B * cols, H, ps)
    table = torch.from_numpy(table_of(rng, B, cols, B * cols)).to(DEV)
    lens = torch.from_numpy(rng.integers(5, cols * ps + 1, B).astype(np.int32)).to(DEV)
    q = queries(B, rows, H * G, 7)
    first = binding.cs_packed_verify_attention(q, pool, table, lens, rows - 1)
    ws = torch.full((1 << 27,), 0xA5, dtype=torch.uint8, device=DEV)   # any contents
    for _ in range(5):
        assert torch.equal(first, binding.cs_packed_verify_attention(q, pool, table, lens, rows - 1, workspace=ws))
