"""Single values through the packed cache that a rounding or a sign step could lose."""
import numpy as np
import pytest
import torch

import serving_reference as ref
from paper_2607_20507_gb300 import binding

pytestmark = pytest.mark.gpu

DEV = "cuda:0"


def host(t):
    return t.detach().cpu().view(torch.uint8).numpy() if t.dtype == torch.float8_e4m3fn else t.detach().cpu().numpy()


@pytest.mark.parametrize("head", [1.0, 0.7, 2.0 ** -70, 2.0 ** 60])
def test_append_keeps_the_sign_of_zeros(head):
    """-0 beside values of every size, in groups that are divided in either way, and tiny values of both signs."""
    H = 2
    rows = np.zeros((1, 7, H, 128), np.float32)
    rows[0, :, :, ::3] = -0.0
    for i, x in enumerate((6.0, 1e-3, 3e38, -5.0, 1e-30, np.nan, 1.0)):
        rows[0, i, :, 1::3] = x
    rows[0, 6, :, 2::6], rows[0, 6, :, 5::6] = -1e-38, 1e-38      # quotients that round to zeros of their sign
    x = torch.from_numpy(rows).bfloat16()
    heads = torch.full((H,), head, device=DEV)
    pool = binding.packed_pool(1, H, 16, DEV, heads, heads)
    table, lens = torch.zeros((1, 1), dtype=torch.int32, device=DEV), torch.full((1,), 7, dtype=torch.int32, device=DEV)
    binding.cs_packed_kv_append(x.to(DEV), (-x).to(DEV), pool, table, lens)
    for t, c, s in ((x, pool.k_codes, pool.k_scales), (-x, pool.v_codes, pool.v_scales)):
        codes, scales = ref.quantise(t.float().numpy(), np.full(H, head))
        np.testing.assert_array_equal(host(s)[0, :, :7], scales[0].swapaxes(0, 1))
        np.testing.assert_array_equal(host(c)[0, :, :7], codes[0].swapaxes(0, 1))


def test_read_rounds_once():
    """Head scales under which a product lies so close to a tie of bf16 that it is one in fp32; the smallest and
    largest products, too."""
    bits = [1037347498, 1041215803, 1043410792, 1045352600, 1032641390, 1032117102, 1032270643, 0x3F800000]
    head = np.concatenate((np.array(bits, np.uint32).view(np.float32),
                           np.array([1.3 * 2.0 ** -118, 1.7 * 2.0 ** -130, 1.1 * 2.0 ** 117], np.float32)))
    H, P, ps = len(head), 4, 256
    gen = torch.Generator().manual_seed(0)
    codes = [torch.randint(0, 256, (P, H, ps, 64), generator=gen, dtype=torch.uint8) for _ in range(2)]
    scales = [torch.randint(0, 0x7F, (P, H, ps, 8), generator=gen, dtype=torch.uint8) for _ in range(2)]
    heads = torch.from_numpy(head).to(DEV)
    pool = binding.PackedPool(*(t.to(DEV) if t.shape[-1] == 64 else t.to(DEV).view(torch.float8_e4m3fn)
                                for t in (codes[0], scales[0], codes[1], scales[1])), heads, heads)
    got = binding.cs_packed_kv_read(pool, torch.arange(P, dtype=torch.int32, device=DEV)[None],
                                    torch.full((1,), P * ps, dtype=torch.int32, device=DEV), P * ps)
    for g, c, s in zip(got, codes, scales):
        want = ref.values(c.numpy(), s.numpy(), head.astype(np.float64)).transpose(0, 2, 1, 3).reshape(1, P * ps, H, 128)
        _, e = np.frexp(want)
        step = np.ldexp(1.0, np.maximum(e - 8, -133))     # of bf16 there
        want = np.rint(want / step) * step                # (exact: powers of two; ties to the even value)
        want = np.where(np.abs(want) > 2.0 ** 128 - 2.0 ** 119, np.copysign(np.inf, want), want)
        np.testing.assert_array_equal(np.abs(g.double().cpu().numpy()), np.abs(want))
        np.testing.assert_array_equal(np.signbit(g.float().cpu().numpy()), np.signbit(want))
