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
