"""Chunk attention where it can go wrong: alignment, rows that are not finite, few keys, workspaces of captured calls."""
import math
import pathlib
import subprocess
import sys

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


def own_workspace(args):
    dims = binding.chunk_attn_dims(args[0], args[1], args[3])
    n = binding.load_library().cs_chunk_attention_workspace_bytes(dims, args[0].shape[0])
    return torch.zeros((n,), dtype=torch.uint8, device=DEV)


def test_one_default_workspace_for_whatever_calls():
    sizes = [([1], [20], 8, 1), ([3, 1], [20, 5], 28, 4), ([300, 7], [0, 100], 32, 32), ([1] * 40, [9] * 40, 64, 8)]
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        all_ = [batch(ns, before, hq, hkv, 16) for ns, before, hq, hkv in sizes]
        got = {binding.chunk_attention_workspace(binding.chunk_attn_dims(a[0], a[1], a[3]), a[0].shape[0], DEV).data_ptr()
               for a in all_}
        held = sum(k[0] == "chunk_attn" and k[2] == side.cuda_stream for k in binding._workspaces)
        for a in all_:
            check(a)
        assert len(got) == 1
        assert sum(k[0] == "chunk_attn" and k[2] == side.cuda_stream for k in binding._workspaces) == held == 1
    side.synchronize()


def test_graphs_of_other_token_counts_after_one_call():
    """Captured after one call of another size, with no fill in the graphs, and replayed in the other order."""
    x = [batch(ns, before, 16, 4, 16, seed=i, junk=False) for i, (ns, before) in enumerate((
        ([1] * 90, [3000 + 37 * b for b in range(90)]), ([1] * 60, [5000] * 60), ([300] * 12, [2000] * 12)))]
    expect = [binding.cs_chunk_attention(*a, workspace=own_workspace(a)) for a in x]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        binding.cs_chunk_attention(*x[0])
    graphs, outs = [], [torch.full_like(e, 3.0) for e in expect]
    before = {k: v.data_ptr() for k, v in binding._workspaces.items()}
    for a, out in zip(x[1:], outs[1:]):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1], stream=side):
            binding.cs_chunk_attention(*a, out=out)
    assert {k: v.data_ptr() for k, v in binding._workspaces.items()} == before
    for i in (1, 0, 1, 0):
        outs[i + 1].fill_(3.0)
        torch.cuda.synchronize()
        graphs[i].replay()
        torch.cuda.synchronize()
        assert torch.equal(outs[i + 1], expect[i + 1])


ALONE = """
import sys
sys.path[:0] = ["tests"]
import torch
from test_gpu_chunk_edges import BY_LAST, DEV, batch, binding, own_workspace
a = batch(*BY_LAST, 16, 4, 16, junk=False)
expect = binding.cs_chunk_attention(*a, workspace=own_workspace(a))
out = torch.full_like(expect, 3.0)
side, pool = torch.cuda.Stream(), torch.cuda.graph_pool_handle()
side.wait_stream(torch.cuda.current_stream())
first, second = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
with torch.cuda.graph(first, pool=pool, stream=side):      # (its memory is free again at the end, with what is in it)
    torch.full((128 << 20,), 7, dtype=torch.uint8, device=DEV)
first.replay()
torch.cuda.synchronize()
with torch.cuda.graph(second, pool=pool, stream=side):     # the process's first call with a default workspace
    %s
for k in range(2):
    for how in ("eager", "replayed"):
        out.fill_(3.0)
        torch.cuda.synchronize()
        if how == "eager":
            with torch.cuda.stream(side):
                binding.cs_chunk_attention(*a, out=out)
        else:
            second.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, expect), (k, how)
print("fine")
"""


@pytest.mark.parametrize("call", ["binding.cs_chunk_attention(*a, out=out)",
                                  "binding.cs_chunk_attention(*a, out=out, stream=side.cuda_stream)"])
def test_a_workspace_made_while_capturing_is_the_graph_s(call):
    """In a process of its own: the first call is a captured one, an eager one on the same stream comes before the first
    replay.  What the graph's memory held before is not zero."""
    r = subprocess.run([sys.executable, "-c", ALONE % call], cwd=pathlib.Path(__file__).parent.parent, capture_output=True,
                       text=True, timeout=300)
    assert r.returncode == 0 and r.stdout.strip() == "fine", r.stderr[-2000:]
