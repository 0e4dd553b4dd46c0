"""Forks, releases and compactions of cache pages against their definitions: every byte, entry and count."""
import numpy as np
import pytest
import torch

import serving_reference as ref
from paper_2607_20507_gb300 import binding

pytestmark = pytest.mark.gpu

DEV = "cuda:0"


class Cache:
    """Pools, table, lengths and counts on both sides."""

    def __init__(self, rng, rows, cols, ps, P, used, shapes=((2, 64), (2, 8))):
        self.ps = ps
        self.lens = np.zeros(rows, np.int32)
        self.table = np.full((rows, cols), -1, np.int32)
        self.refs = np.zeros(P, np.int32)
        order = list(rng.permutation(P))
        for r in range(used):
            self.lens[r] = rng.integers(0, cols * ps + 1)
            for j in range(-(-int(self.lens[r]) // ps)):
                if not order:
                    self.lens[r] = j * ps
                    break
                self.table[r, j] = order.pop()
                self.refs[self.table[r, j]] += 1
        self.pools = [rng.integers(0, 256, (P, s[0], ps, s[1]), dtype=np.uint8) for s in shapes]
        self.dev()

    def dev(self):
        self.d_pools = [torch.from_numpy(p.copy()).to(DEV) for p in self.pools]
        self.d_table, self.d_lens, self.d_refs = (torch.from_numpy(a.copy()).to(DEV)
                                                  for a in (self.table, self.lens, self.refs))

    def same(self):
        np.testing.assert_array_equal(self.d_table.cpu().numpy(), self.table)
        np.testing.assert_array_equal(self.d_lens.cpu().numpy(), self.lens)
        np.testing.assert_array_equal(self.d_refs.cpu().numpy(), self.refs)
        for d, p in zip(self.d_pools, self.pools):
            np.testing.assert_array_equal(d.cpu().numpy(), p)

    def fork(self, src, dst, room=0):
        got = binding.cs_kv_fork(self.d_pools, self.d_table, self.d_lens, self.d_refs, ints(src), ints(dst), self.ps, room)
        want = ref.fork(self.pools, self.table, self.lens, self.refs, src, dst, self.ps, room)
        np.testing.assert_array_equal(got.cpu().numpy(), want)
        self.same()
        return want

    def release(self, rows, keep):
        binding.cs_kv_release(self.d_table, self.d_lens, self.d_refs, ints(rows), ints(keep), self.ps)
        ref.release(self.table, self.lens, self.refs, rows, keep, self.ps)
        self.same()

    def compact(self):
        got = binding.cs_kv_compact(self.d_pools, self.d_table, self.d_refs)
        assert int(got) == ref.compact(self.pools, self.table, self.refs)
        self.same()


def ints(v):
    return torch.as_tensor(np.asarray(v), dtype=torch.int32).to(DEV)


@pytest.mark.parametrize("ps", [1, 8, 16, 64, 256])
@pytest.mark.parametrize("room", [0, 1, 40, 10 ** 6])
def test_fork(ps, room):
    rng = np.random.default_rng(ps + room)
    c = Cache(rng, 12, 5, ps, 90, 4)
    c.lens[3] = min(c.lens[3], c.lens[3] // ps * ps)      # a full last page
    c.table[3, c.lens[3] // ps:] = -1
    c.refs[:] = 0
    for p in c.table[c.table >= 0]:
        c.refs[p] += 1
    c.dev()
    c.fork([0, 0, 1, 2, 3, 3, -1], [4, 5, 6, 7, 8, 9, 10], room)


def test_fork_runs_out_of_pages():
    rng = np.random.default_rng(1)
    c = Cache(rng, 40, 6, 16, 24, 3)
    done = c.fork([0, 1, 2, -1] * 8, list(range(3, 35)), room=33)
    assert 0 < done.sum() < len(done)
    c.release([3, 4, 5, 6], [0, 0, 0, 0])
    c.fork([-1, -1], [36, 37], room=17)


def test_fork_of_rows_that_are_none():
    rng = np.random.default_rng(2)
    c = Cache(rng, 8, 4, 16, 64, 3)
    c.table[1, 0], c.table[2, :2] = 1 << 20, (-9, 64)   # entries outside the pool are carried along
    c.lens[1:3] = (10, 35)
    c.dev()
    c.fork([0, 8, -2, 1, 2, 0, 0, 100], [3, 4, 5, 6, 7, -1, 8, 99])


def test_many_forks_of_one_row():
    rng = np.random.default_rng(3)
    c = Cache(rng, 1500, 3, 16, 4000, 1)
    c.lens[0] = 37
    c.refs[:] = 0
    c.table[0] = (17, 3, 3999)
    c.refs[[17, 3, 3999]] = 1
    c.dev()
    c.fork([0] * 1400, list(range(1, 1401)), room=5)
    c.release(list(range(1, 1401, 2)), [0] * 700)
    c.compact()


@pytest.mark.parametrize("P", [1, 15, 16, 17, 4095, 4096, 4097, 20000])
@pytest.mark.parametrize("share", [0.0, 0.03, 0.5, 0.97, 1.0])
def test_compact_any_pool(P, share):
    """Pools of one page to several tiles of counts, empty to full."""
    rng = np.random.default_rng(P + int(100 * share))
    c = Cache(rng, 7, 11, 8, P, 0, shapes=((1, 2),))
    on = rng.random(P) < share if 0 < share < 1 else np.full(P, bool(share))
    c.refs[:] = np.where(on, rng.integers(1, 4, P), 0)
    ids = np.flatnonzero(on)
    if len(ids):
        c.table[:] = np.where(rng.random(c.table.shape) < 0.8, rng.choice(ids, c.table.shape), c.table)
    c.table[0, :3] = (P, 1 << 30, -(1 << 31))
    c.dev()
    c.compact()
    c.compact()     # nothing is left to move


def test_release_keeps_a_prefix():
    rng = np.random.default_rng(4)
    c = Cache(rng, 10, 6, 16, 80, 8)
    c.fork([0, 1], [8, 9], room=20)
    c.release([0, 1, 2, 3, 4, 8, 9, 10, -1], [16, 17, 10 ** 9, -5, 0, 1, int(c.lens[9]) + 20, 3, 3])


def test_life_of_a_cache():
    """Rounds of forks, releases and compactions, in which no count is lost."""
    rng = np.random.default_rng(5)
    c = Cache(rng, 30, 8, 16, 150, 5)
    for _ in range(12):
        used, idle = np.flatnonzero(c.lens > 0), np.flatnonzero(c.lens == 0)
        n = min(len(idle), 6)
        if n:
            c.release(idle[:n], [0] * n)
            c.fork(rng.choice(np.append(used, -1), n), rng.permutation(idle[:n]), int(rng.integers(0, 40)))
        used = np.flatnonzero(c.lens > 0)
        k = int(rng.integers(0, len(used) + 1))
        c.release(rng.permutation(used)[:k], rng.integers(0, 100, k))
        if rng.random() < 0.5:
            c.compact()
        counts = np.bincount(c.table[c.table >= 0], minlength=150)
        np.testing.assert_array_equal(counts, c.refs)


def test_bf16_pools_of_many_layers():
    """Pools of several shapes and types, as a model of many layers has them."""
    rng = np.random.default_rng(6)
    c = Cache(rng, 9, 4, 16, 50, 3, shapes=((2, 256), (2, 256), (1, 1), (3, 80)) * 20)
    c.fork([0, 1, 2], [3, 4, 5], 3)
    c.release([0, 4], [0, 0])
    c.compact()


def test_copies_past_32_bits():
    """A pool of more than 2^32 bytes whose last page moves to its first."""
    P, ps = 4200, 16
    pool = torch.zeros(P, 1 << 20, dtype=torch.uint8, device=DEV)
    pool[P - 1] = torch.arange(1 << 20, device=DEV).to(torch.uint8)
    refs = torch.zeros(P, dtype=torch.int32, device=DEV)
    refs[P - 1] = 1
    table = torch.tensor([[P - 1, -1]], dtype=torch.int32, device=DEV)
    live = binding.cs_kv_compact([pool], table, refs)
    assert int(live) == 1 and table[0, 0] == 0 and refs[0] == 1 and refs[P - 1] == 0
    assert torch.equal(pool[0], pool[P - 1])


def test_on_a_side_stream():
    rng = np.random.default_rng(7)
    c = Cache(rng, 20, 6, 16, 200, 6)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        c.fork([0, 1, 2, 3], [6, 7, 8, 9], 30)
        c.release([0, 7], [0, 5])
        c.compact()


def test_binding_refuses():
    rng = np.random.default_rng(8)
    c = Cache(rng, 4, 3, 16, 20, 2)
    args = dict(pools=c.d_pools, page_table=c.d_table, ctx_lens=c.d_lens, ref_counts=c.d_refs, src=ints([0]), dst=ints([2]),
                page_size=16)
    for bad, kind in ((dict(src=ints([0, 1])), ValueError), (dict(src=ints([0]).long()), TypeError),
                      (dict(page_size=0), binding.CacheSpecError), (dict(room=-1), binding.CacheSpecError),
                      (dict(pools=[c.d_pools[0][:10]]), ValueError), (dict(ref_counts=c.d_refs.cpu()), ValueError),
                      (dict(pools=[torch.zeros(20, 3, dtype=torch.uint8, device=DEV)]), binding.CacheSpecError),
                      (dict(pools=[c.d_pools[0].transpose(1, 2)]), ValueError), (dict(ctx_lens=c.d_lens[:2]), ValueError),
                      (dict(workspace=torch.zeros(256, dtype=torch.uint8, device=DEV)), binding.CacheSpecError),
                      (dict(pools=c.d_pools * 65), binding.CacheSpecError)):
        with pytest.raises(kind):
            binding.cs_kv_fork(**{**args, **bad})
    with pytest.raises(ValueError):
        binding.cs_kv_release(c.d_table, c.d_lens, c.d_refs, ints([0]), ints([0, 1]), 16)
    with pytest.raises(ValueError):
        binding.cs_kv_compact(c.d_pools, c.d_table[0], c.d_refs)
    c.same()
    assert binding.cs_kv_fork(**{**args, "src": ints([]), "dst": ints([])}).shape == (0,)
    binding.cs_kv_release(c.d_table, c.d_lens, c.d_refs, ints([]), ints([]), 16)
    c.same()
