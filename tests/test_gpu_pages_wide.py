"""Page operations whose sums and sizes pass 32 bits."""
import pytest
import torch

from paper_2607_20507_gb300 import binding

pytestmark = pytest.mark.gpu

DEV = "cuda:0"


def test_forks_that_ask_for_more_than_2_31_pages():
    """1024 requests of 2^21 pages each: the pool holds those of the first, and no other gets any."""
    rows, cols, ps = 1024, 1 << 21, 16
    P = cols + 5
    pool = torch.arange(P * 16, dtype=torch.int32, device=DEV).view(torch.uint8).view(P, -1)
    before = pool.clone()
    table = torch.zeros((rows, cols), dtype=torch.int32, device=DEV)
    lens = torch.full((rows,), 7, dtype=torch.int32, device=DEV)
    refs = torch.zeros(P, dtype=torch.int32, device=DEV)
    dst = torch.arange(rows, dtype=torch.int32, device=DEV)
    done = binding.cs_kv_fork([pool], table, lens, refs, torch.full_like(dst, -1), dst, ps, cols * ps)
    assert done.tolist() == [1] + [0] * (rows - 1)
    assert torch.equal(table[0], torch.arange(cols, dtype=torch.int32, device=DEV))
    assert all(bool((table[r:r + 64] == -1).all()) for r in range(1, rows, 64))
    assert not lens.any() and torch.equal(pool, before)
    assert bool((refs[:cols] == 1).all()) and not refs[cols:].any()
