"""Log probabilities, entropies and top alternatives against the definition in 64 bits."""
import numpy as np
import pytest
import torch

import serving_reference as ref
from paper_2607_20507_gb300 import binding

pytestmark = pytest.mark.gpu

DEV = "cuda:0"


def check(logits, tokens, T=1.0, n_top=0):
    """logits: a device tensor [N, V], any row stride."""
    got = binding.cs_logprobs(logits, torch.as_tensor(tokens, dtype=torch.int32).to(DEV), T, n_top)
    z = logits.double().cpu().numpy()
    lp, ent, ids, top = ref.logprobs(z, np.asarray(tokens), T, n_top)
    with np.errstate(over="ignore"):   # (what passes the outputs' type is -inf in it)
        lp, top = (x.astype(np.float32).astype(np.float64) for x in (lp, top))
    g = [t.cpu().numpy() for t in got]
    np.testing.assert_array_equal(g[2], ids)
    for a, b in ((g[0], lp), (g[3], top)):
        np.testing.assert_array_equal(np.isneginf(a), np.isneginf(b))
        on = np.isfinite(b)
        # (z - max) log2(e) / T to 2^-22 of itself, the sum's logarithm to 1e-5
        assert (np.abs(a[on] - b[on]) <= 1e-5 + 2.0 ** -21 * np.abs(b[on])).all(), np.abs(a[on] - b[on]).max()
    # sums of weights times their logarithms, whose sizes add up to about lse + H
    assert (np.abs(g[1] - ent) <= 2e-5 * (1 + np.log(z.shape[1]) + ent)).all(), np.abs(g[1] - ent).max()
    assert (g[1] >= 0).all()
    return got


def normal(N, V, seed, dtype=torch.float32, size=3.0):
    return (torch.randn(N, V, generator=torch.Generator().manual_seed(seed)) * size).to(dtype).to(DEV)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V", [1, 2, 7, 31, 33, 255, 1000, 4096, 8191, 32001, 128256])
@pytest.mark.parametrize("n_top", [0, 1, 5, 32])
def test_vocabularies(dtype, V, n_top):
    N = 5
    tokens = np.random.default_rng(V).integers(0, V, N)
    check(normal(N, V, V + n_top, dtype), tokens, 0.8, n_top)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("N,V", [(1, 256000), (3, 300007), (700, 1003), (2, 1 << 21)])
def test_few_and_many_rows(dtype, N, V):
    tokens = np.random.default_rng(N).integers(0, V, N)
    check(normal(N, V, N + V, dtype), tokens, 1.0, 20)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V,stride,offset", [(1000, 1024, 0), (999, 1001, 1), (5003, 5004, 3), (4096, 4097, 0), (40, 64, 7)])
def test_rows_that_lie_apart(dtype, V, stride, offset):
    """Padded vocabularies and rows that start at any element; what lies between them is never read."""
    N = 6
    flat = torch.full((offset + N * stride,), float("nan"), dtype=dtype, device=DEV)
    view = flat[offset:].view(N, stride)[:, :V]
    view.copy_(normal(N, V, V, dtype))
    check(view, np.arange(N) * 7 % V, 1.3, 8)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_tokens_that_are_none(dtype):
    """Negative tokens skip their row (which may hold anything); tokens past the vocabulary have no probability."""
    z = normal(8, 5000, 3, dtype)
    z[1] = float("nan")
    z[6] = float("inf")
    tokens = torch.tensor([3, -1, 4999, 5000, 2 ** 31 - 1, 0, -2 ** 31, -1], dtype=torch.int32)
    lp, ent, ids, top = binding.cs_logprobs(z, tokens.to(DEV), 1.0, 4)
    for r in (1, 6, 7):
        assert lp[r] == -float("inf") and ent[r] == 0 and (ids[r] == -1).all() and (top[r] == -float("inf")).all()
    keep = [0, 2, 3, 4, 5]
    check(z[keep], tokens[keep].numpy(), 1.0, 4)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_masked_logits(dtype):
    """-inf from none to all of a row; fewer left than alternatives are asked for."""
    V = 3001
    z = normal(9, V, 4, dtype)
    z[1, 1:] = -float("inf")
    z[2, :-1] = -float("inf")
    z[3] = -float("inf")
    z[4, ::2] = -float("inf")
    z[5, 10:] = -float("inf")
    z[6, :2990] = -float("inf")
    z[7, 1500:] = -float("inf")
    z[8, :] = -float("inf")
    z[8, 77] = torch.finfo(dtype).min
    check(z, [5, 0, V - 1, 4, 6, 20, 2995, 3, 77], 0.7, 20)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_lowest_and_largest_values(dtype):
    lo, hi = torch.finfo(dtype).min, torch.finfo(dtype).max
    V = 2000
    z = torch.zeros(6, V, dtype=dtype, device=DEV)
    z[0] = lo                     # all masked by the lowest value: uniform
    z[1] = lo
    z[1, 5:9] = 1.0
    z[2] = hi
    z[3, ::2] = lo
    z[3, 1::2] = hi               # differences past the type
    z[4, 3] = 30000.0
    z[5] = normal(1, V, 5, dtype, 1e30)[0]
    check(z, [0, 6, 1999, 1, 3, 17], 1.0, 6)
    check(z[:3], [3, 100, 0], 1e-30, 6)
    check(z[:5], [0, 6, 1999, 1, 4], 100.0, 3)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("order", ["equal", "up", "down", "few", "late", "blocks", "zeros"])
@pytest.mark.parametrize("V", [700, 70001])
def test_orders_and_ties(dtype, order, V):
    """Rows on which a running selection has most to do, and ties, which go to the lowest id."""
    v = torch.arange(V, device=DEV)
    z = {"equal": torch.zeros(V, device=DEV) - 2.5, "up": v * 1e-3, "down": -v * 1e-3, "few": (v % 3).float(),
         "late": (v >= V - 40).float() * (v % 7), "blocks": (v // 256 % 19).float(),
         "zeros": torch.where(v % 2 == 0, 0.0, -0.0)}[order]
    check(z.to(dtype).repeat(2, 1), [0, V - 1], 1.0, 32)


@pytest.mark.parametrize("T", [1e-3, 0.1, 0.5, 1.0, 7.3, 1e4])
def test_temperatures(T):
    check(normal(4, 9001, 6), [0, 1, 2, 9000], T, 10)


def test_after_an_acceptance_step():
    """The emitted tokens of cs_spec_accept under the target's rows; the positions past them are skipped."""
    gen = torch.Generator().manual_seed(7)
    B, k, V = 6, 4, 4001
    target = (torch.randn(B, k + 1, V, generator=gen) * 3).bfloat16().to(DEV)
    draft = (target[:, :k].float() + 0.5 * torch.randn(B, k, V, generator=gen).to(DEV)).bfloat16()
    tokens = torch.randint(0, V, (B, k), generator=gen).int().to(DEV)
    tokens[:, 0] = target[:, 0].argmax(1).int()
    out, n = binding.cs_spec_accept(target, draft, tokens, torch.rand(B, k + 1, generator=gen).to(DEV), 0.8)
    lp, _, _, _ = check(target.view(-1, V), out.view(-1).cpu().numpy(), 0.8, 3)
    skipped = torch.arange(k + 1, device=DEV)[None] > n[:, None]
    assert (lp.view(B, k + 1)[skipped] == -float("inf")).all()
    assert torch.isfinite(lp.view(B, k + 1)[~skipped]).all()


def test_same_bits_on_any_stream_and_in_a_graph():
    z, tok = normal(37, 50021, 8, torch.bfloat16), torch.arange(37, dtype=torch.int32, device=DEV)
    first = binding.cs_logprobs(z, tok, 0.9, 12)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        again = binding.cs_logprobs(z * 1.0, tok, 0.9, 12)
    side.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        graphed = binding.cs_logprobs(z, tok, 0.9, 12)
    g.replay()
    torch.cuda.synchronize()
    for a, b, c in zip(first, again, graphed):
        assert torch.equal(a, b) and torch.equal(a, c)


def test_binding_refuses():
    z, tok = normal(3, 50, 9), torch.zeros(3, dtype=torch.int32, device=DEV)
    for bad, kind in ((dict(logits=z.half()), TypeError), (dict(logits=z[0]), ValueError), (dict(logits=z.cpu()), ValueError),
                      (dict(logits=z.t()), ValueError), (dict(tokens=tok.long()), TypeError), (dict(tokens=tok[:2]), ValueError),
                      (dict(temperature=0.0), binding.CacheSpecError), (dict(temperature=float("inf")), binding.CacheSpecError),
                      (dict(temperature=float("nan")), binding.CacheSpecError), (dict(n_top=33), binding.CacheSpecError),
                      (dict(n_top=-1), binding.CacheSpecError)):
        with pytest.raises(kind):
            binding.cs_logprobs(**{**dict(logits=z, tokens=tok), **bad})
    lp, ent, ids, top = binding.cs_logprobs(z[:0], tok[:0], 1.0, 2)
    assert lp.shape == ent.shape == (0,) and ids.shape == top.shape == (0, 2)
