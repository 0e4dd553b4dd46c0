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


def fine(args):
    """The framework's bound of attention outputs; and the output's rounding (half a step, 2^-8 of the value) with scores,
    weights and sums in 16 bits and more: weights of two bf16 terms are off by at most 2^-16 of themselves, fp32 scores of
    128 products by 128 * 2^-24 of some 10, sums of up to 4000 weights by a good deal less than 4000 * 2^-24: 2^-11
    together.  (Weights of one bf16 term are off by up to 2^-8.)"""
    out = binding.cs_chunk_attention(*args)
    expect, size = ref.attention(*args)
    off = (out.double() - expect).abs()
    assert not (off > 2e-3 + 1e-2 * expect.abs()).any()
    assert not (off > 1.01 * 2.0 ** -8 * expect.abs() + 2.0 ** -11 * size).any()


@pytest.mark.parametrize("L", [1, 2, 3, 5, 9, 17, 33, 128, 129])
@pytest.mark.parametrize("hq,hkv", [(8, 2), (32, 1)])
def test_weights_of_few_keys_are_not_rounded_to_bf16(L, hq, hkv):
    fine(batch([1] * 150, [L - 1] * 150, hq, hkv, 16, seed=L))


def test_the_first_rows_of_prompts():
    fine(batch([17, 40, 130, 9] * 12, [0] * 48, 16, 4, 16, seed=5))


@pytest.mark.parametrize("ns,before", [WHOLE, BY_KERNEL, BY_LAST, ([1] * 60 + [90], [500] * 60 + [3500])])
def test_weights_of_longer_contexts_and_of_cut_blocks(ns, before):
    fine(batch(ns, before, 16, 4, 16, seed=9, junk=False))


@pytest.mark.parametrize("heavy", [2, 3, 7])
@pytest.mark.parametrize("growing", [False, True])
def test_a_few_keys_that_outweigh_the_others(heavy, growing):
    """Scores of a few keys anywhere in a long context stand 16 above the others', all alike or each above the last."""
    ns, before = [1, 200, 3], [5000, 1200, 2600]
    q, k, v, table, lens, starts = batch(ns, before, 8, 2, 16, seed=heavy, junk=False)
    q[:, :, 0] = 16.0
    k[..., 0] = 0.0
    gen = torch.Generator().manual_seed(heavy)
    for b, L in enumerate(lens.tolist()):
        for i, j in enumerate(sorted(torch.randperm(before[b], generator=gen)[:heavy].tolist())):
            # 16 * 11.25 / sqrt(128) = 15.9; growing: a step of 0.5 is 0.7 of a score
            k[table[b, j // 16], :, j % 16, 0] = 11.25 + (0.5 * i if growing else 0)
    fine((q, k, v, table, lens, starts))


@pytest.mark.parametrize("ns,before", [WHOLE, BY_KERNEL, BY_LAST])
@pytest.mark.parametrize("bad", [math.nan, math.inf])
def test_rows_that_are_not_finite_stay_so_and_alone(ns, before, bad):
    """In whole blocks and in either join: one entry of a few query rows is NaN, or infinite (scores of both signs)."""
    q, k, v, table, lens, starts = batch(ns, before, 16, 4, 16, seed=3, junk=False)
    clean = binding.cs_chunk_attention(q, k, v, table, lens, starts)
    hit = torch.zeros(clean.shape[:2], dtype=torch.bool, device=DEV)
    for b, n in enumerate(ns):
        if n:
            hit[int(starts[b]) + n // 2, (5 * b + 3) % 16] = True
            hit[int(starts[b]) + n - 1, 15] = True
    q = q.contiguous()
    q[..., 7][hit] = bad
    got = binding.cs_chunk_attention(q, k, v, table, lens, starts)
    assert torch.equal(got[~hit], clean[~hit])
    assert torch.isnan(got[hit]).all()
