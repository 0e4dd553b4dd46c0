"""Packed attention over many short contexts: a CTA takes many spans of one to a few tiles, so that every buffer
changes hands from tile to tile.  Against the definition in 64 bits."""
import numpy as np
import pytest
import torch

from paper_2607_20507_gb300 import binding

pytestmark = pytest.mark.gpu
DEV = "cuda:0"

E2M1 = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float64)


def values(codes, scales):
    """fp64 [P, H, ps, 128] of codes [P, H, ps, 64] and e4m3 scales [P, H, ps, 8]."""
    c = torch.stack((codes & 15, codes >> 4), -1).flatten(-2).long()
    v = E2M1.to(DEV)[c & 7] * torch.where(c > 7, -1.0, 1.0).double()
    return v * scales.double().repeat_interleave(16, -1)


@pytest.mark.parametrize("rows,G", [(1, 4), (5, 4), (4, 7), (8, 4), (12, 4), (5, 8), (7, 7), (7, 8), (9, 8), (16, 5),
                                    (13, 8), (17, 8)])
@pytest.mark.parametrize("B,lo,hi", [(229, 80, 450), (300, 1, 129), (64, 250, 700)])
def test_many_short_spans(rows, G, B, lo, hi):
    rng = np.random.default_rng(rows * 100 + G + B)
    H, ps = 4, 16
    cols = (hi + ps - 1) // ps
    P = B * cols + 3
    g = torch.Generator(device=DEV).manual_seed(rows + B)
    pool = binding.packed_pool(P, H, ps, DEV)
    for codes, scales in ((pool.k_codes, pool.k_scales), (pool.v_codes, pool.v_scales)):
        codes.copy_(torch.randint(0, 256, codes.shape, generator=g, device=DEV, dtype=torch.uint8))
        scales.view(torch.uint8).copy_(torch.randint(0x28, 0x38, scales.shape, generator=g, device=DEV,
                                                     dtype=torch.uint8))
    table = torch.from_numpy(rng.permutation(P)[:B * cols].reshape(B, cols).astype(np.int32)).to(DEV)
    lens = torch.from_numpy(rng.integers(lo, hi + 1, B).astype(np.int32)).to(DEV)
    # a row's size differs from span to span: a scale taken for another's shows
    q = torch.randn((B, rows, H * G, 128), generator=g, device=DEV)
    q = (q * torch.rand((B, 1, H, 1, 1), generator=g, device=DEV).mul(4).exp2().expand(B, 1, H, G, 1).reshape(
        B, 1, H * G, 1) * 0.2).to(torch.bfloat16)
    out = binding.cs_packed_verify_attention(q, pool, table, lens, rows - 1).double()
    n = cols * ps
    K, V = (values(c, s)[table.long()].transpose(1, 2).reshape(B, H, n, 128)
            for c, s in ((pool.k_codes, pool.k_scales), (pool.v_codes, pool.v_scales)))
    z = torch.einsum("bihgd,bhjd->bhigj", q.double().view(B, rows, H, G, 128), K) * 128 ** -0.5
    last = lens.long()[:, None] - rows + torch.arange(rows, device=DEV)            # [B, rows]
    seen = torch.arange(n, device=DEV)[None, None] <= last[..., None]              # [B, rows, n]
    z = z.masked_fill(~seen[:, None, :, None], -float("inf"))
    w = torch.where(last[:, None, :, None, None] < 0, torch.zeros((), device=DEV, dtype=torch.float64),
                    (z - z.amax(-1, keepdim=True).clamp(min=-1e300)).exp())
    total = w.sum(-1, keepdim=True)
    w = w / torch.where(total > 0, total, 1.0)
    expect = torch.einsum("bhigj,bhjd->bihgd", w, V).reshape(B, rows, H * G, 128)
    size = torch.einsum("bhigj,bhjd->bihgd", w, V.abs()).reshape(B, rows, H * G, 128)
    # the output's rounding to bf16 (2^-8 of it at most), the weights' to 11 bits, fp32 sums and
    # exponents (scores up to some hundreds: 2^-15)
    bad = ~((out - expect).abs() <= 1.01 * 2.0 ** -8 * expect.abs() + (2.0 ** -11 + 2.0 ** -15) * size + 1e-37)
    assert not bad.any(), (int(bad.sum()), bad.nonzero()[:4].tolist())
