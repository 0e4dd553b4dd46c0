"""Chunk attention where it can go wrong: alignment, rows that are not finite, few keys, workspaces of captured calls."""
import math

import pytest
import torch

import ragged_reference as ref
from paper_2607_20507_gb300 import binding
from test_gpu_chunk import batch, check

pytestmark = pytest.mark.gpu

DEV = "cuda:0"

# calls whose blocks are whole; cut, and joined by a second kernel; cut, and joined by whoever comes last
WHOLE, BY_KERNEL, BY_LAST = ([5, 140, 0, 1], [50, 20, 7, 300]), ([1, 70], [9000, 2500]), ([300] * 12, [2000] * 12)


def shifted(t):
    """The same tensor 16 bytes behind a 32-byte boundary."""
    x = torch.empty((t.numel() + 24,), dtype=t.dtype, device=t.device)
    at = next(i for i in range(0, 24, 8) if (x.data_ptr() + 2 * i) % 32 == 16)
    y = x[at:at + t.numel()].view(t.shape)
    y.copy_(t)
    assert y.data_ptr() % 32 == 16
    return y


@pytest.mark.parametrize("ns,before", [WHOLE, BY_KERNEL, BY_LAST, ([6, 40], [-4, -38])])
@pytest.mark.parametrize("which", ["out", "q", "pages"])
def test_arrays_aligned_to_16_bytes(ns, before, which):
    q, k, v, table, lens, starts = batch(ns, [max(p, 0) for p in before], 16, 4, 16, junk=False)
    lens = torch.tensor([n + p for n, p in zip(ns, before)], dtype=torch.int32, device=DEV)
    expect = check((q, k, v, table, lens, starts))
    q = q.contiguous()
    out = torch.full(q.shape, 3.0, dtype=torch.bfloat16, device=DEV)
    if which == "out":
        out = shifted(out)
    elif which == "q":
        q = shifted(q)
    else:
        k, v = shifted(k), shifted(v)
    got = binding.cs_chunk_attention(q, k, v, table, lens, starts, out=out)
    assert got is out and torch.equal(got, expect)
