"""Forks and compactions of caches with more arrays than one call takes, and forks past a shortage."""
import importlib.util
import os

import numpy as np
import pytest
import torch

import serving_reference as ref
from paper_2607_20507_gb300 import binding

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
M = binding.CS_MAX_PAGE_POOLS
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def ints(v):
    return torch.as_tensor(np.asarray(v), dtype=torch.int32).to(DEV)


@pytest.mark.parametrize("count", [M, M + 1, 330])     # 330: a model of 82 layers, and two arrays of its own
@pytest.mark.parametrize("own_workspace", [False, True])
def test_every_array_follows_the_table(count, own_workspace):
    rng = np.random.default_rng(count)
    rows, cols, ps, P = 12, 5, 16, 60
    table, lens, refs = np.full((rows, cols), -1, np.int32), np.zeros(rows, np.int32), np.zeros(P, np.int32)
    order = list(rng.permutation(P))
    for r in range(4):
        lens[r] = rng.integers(1, cols * ps + 1)
        for j in range(-(-int(lens[r]) // ps)):
            table[r, j] = order.pop()
            refs[table[r, j]] = 1
    table[2, lens[2] // ps if lens[2] % ps else 0] = P      # a page outside the pool: carried along
    pools = [rng.integers(0, 256, (P, 16 * (1 + i % 9 * (1 + i % 5 * 40))), dtype=np.uint8) for i in range(count)]
    d_pools = [torch.from_numpy(p.copy()).to(DEV) for p in pools]
    d_table, d_lens, d_refs = ints(table), ints(lens), ints(refs)
    ws = torch.empty(1 << 16, dtype=torch.uint8, device=DEV) if own_workspace else None

    def same():
        for d, h in ((d_table, table), (d_lens, lens), (d_refs, refs), *zip(d_pools, pools)):
            np.testing.assert_array_equal(d.cpu().numpy(), h)

    src, dst = [0, 1, 1, 2, 3, -1], [4, 5, 6, 7, 8, 9]
    done = binding.cs_kv_fork(d_pools[:M], d_table, d_lens, d_refs, ints(src), ints(dst), ps, 3, workspace=ws)
    for i in range(M, count, M):
        binding.cs_kv_fork_more(d_pools[i:i + M], d_table, d_refs, len(src), workspace=ws)
    np.testing.assert_array_equal(done.cpu().numpy(), ref.fork(pools, table, lens, refs, src, dst, ps, 3))
    same()
    gone = [0, 3, 5]
    binding.cs_kv_release(d_table, d_lens, d_refs, ints(gone), ints([0] * 3), ps)
    ref.release(table, lens, refs, gone, [0] * 3, ps)
    live = binding.cs_kv_compact(d_pools[:M], d_table, d_refs, workspace=ws)
    for i in range(M, count, M):
        binding.cs_kv_compact_more(d_pools[i:i + M], d_table, d_refs, workspace=ws)
    assert int(live) == ref.compact(pools, table, refs)
    same()


def test_a_workspace_that_lists_no_pages():
    """Entries of a list that are no pages (here -1: what a workspace of 0xff bytes holds) are left out."""
    pool = torch.arange(64, dtype=torch.int32, device=DEV).view(torch.uint8).view(16, 16).clone()
    before = pool.clone()
    table, refs = torch.full((2, 4), -1, dtype=torch.int32, device=DEV), torch.zeros(16, dtype=torch.int32, device=DEV)
    ws = torch.full((1 << 16,), 0xFF, dtype=torch.uint8, device=DEV)
    binding.cs_kv_fork_more([pool], table, refs, 100, workspace=ws)
    binding.cs_kv_compact_more([pool], table, refs, workspace=ws)
    assert torch.equal(pool, before)


def test_the_example_with_a_model_of_many_layers():
    """40 layers, 160 arrays: what the rows hold in every layer survives fork, release and compaction."""
    spec = importlib.util.spec_from_file_location("packed_serving", os.path.join(ROOT, "examples", "packed_serving.py"))
    ex = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(ex)
    prompt, room, ps = 45, 20, 16
    cols = (prompt + room) // ps + 2
    s = ex.Server(ex.StandIn(40, 4, 2, 501, torch.device(DEV)), 4, 4 * cols, ps, cols)
    assert len(s.page_pools) > M and s.prefill(0, prompt).all()
    read = lambda row: [torch.cat(binding.cs_packed_kv_read(p, s.table[row:row + 1], s.lens[row:row + 1], prompt))  # noqa: E731
                        for p in s.pools]
    want = read(0)
    assert all(bool(w.any()) for w in want)
    assert s.fork([0, 0, 0], [1, 2, 3], room).all()
    for row in (1, 2, 3):
        assert all(torch.equal(a, b) for a, b in zip(read(row), want))
    s.release([0, 1, 2])
    assert int(s.compact()) == -(-(prompt + room) // ps)
    assert all(torch.equal(a, b) for a, b in zip(read(3), want))


@pytest.mark.parametrize("lens,free,want", [((9, 8), 0, (0, 0)), ((8, 9), 0, (1, 0)), ((8, 9, 8, 16, 9), 1, (1, 1, 1, 1, 0)),
                                            ((9, 17, 8, 8), 1, (1, 0, 0, 0))])
def test_from_a_shortage_on_no_row_is_forked(lens, free, want):
    """Rows of whole pages ask for none, but not past a request that went without."""
    ps, cols, n = 8, 3, len(lens)
    used = [-(-L // ps) for L in lens]
    P = sum(used) + free
    table, at = np.full((2 * n, cols), -1, np.int32), 0
    for r, u in enumerate(used):
        table[r, :u] = range(at, at + u)
        at += u
    lens = np.array(lens + (0,) * n, np.int32)
    refs = (np.arange(P) < at).astype(np.int32)
    pools = [np.random.default_rng(n).integers(0, 256, (P, 32), dtype=np.uint8)]
    dev = [torch.from_numpy(a.copy()).to(DEV) for a in (pools[0], table, lens, refs)]
    src, dst = list(range(n)), list(range(n, 2 * n))
    done = binding.cs_kv_fork([dev[0]], *dev[1:], ints(src), ints(dst), ps)
    assert tuple(done.tolist()) == want == tuple(ref.fork(pools, table, lens, refs, src, dst, ps, 0))
    for d, h in zip(dev, (pools[0], table, lens, refs)):
        np.testing.assert_array_equal(d.cpu().numpy(), h)
