"""Packed attention whose query rows lie more than 2^31 elements apart."""
import pytest
import torch

from paper_2607_20507_gb300 import binding

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
E2M1 = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


@pytest.mark.parametrize("G", [1, 2])
def test_rows_past_32_bits(G):
    """2^20 query heads and 16 drafts: the last row starts 2^31 elements past the first.  Keys of 0 weigh the same,
    so row i is the mean of the values that it sees."""
    Hq, R, ps = 1 << 20, 17, 8
    H = Hq // G     # 17 query rows a KV head (one form), or 34 (the other)
    g = torch.Generator(device=DEV).manual_seed(G)
    pool = binding.packed_pool(1, H, ps, DEV)
    pool.v_codes.random_(0, 256, generator=g)
    pool.v_scales.view(torch.uint8).fill_(0x38)     # 1
    q = torch.ones((1, R, Hq, 128), dtype=torch.bfloat16, device=DEV)
    one = torch.zeros((1, 1), dtype=torch.int32, device=DEV)
    out = binding.cs_packed_verify_attention(q, pool, one, one.view(1) + ps, R - 1).view(R, H, G, 128)
    del q
    for i in range(R):
        n = ps - R + 1 + i      # keys that row i sees
        if n <= 0:
            assert not out[i].any()
            continue
        c = pool.v_codes[0, :, :n]
        expect = torch.zeros((H, 64, 2), device=DEV)
        size = torch.zeros_like(expect)
        for j in range(n):      # sums of multiples of 0.5: exact
            for half, code in enumerate((c[:, j] & 15, c[:, j] >> 4)):
                a = E2M1.to(DEV)[(code & 7).int()]
                expect[:, :, half] += torch.where(code > 7, -a, a)
                size[:, :, half] += a
        expect, size = expect.view(H, 1, 128) / n, size.view(H, 1, 128) / n
        # the output's rounding to bf16 (2^-8 of it at most), the weights' to 11 bits, fp32 sums
        bad = ~((out[i].float() - expect).abs() <= 1.01 * 2.0 ** -8 * expect.abs() + (2.0 ** -11 + 2.0 ** -15) * size)
        assert not bad.any(), (i, int(bad.sum()))
