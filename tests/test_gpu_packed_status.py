"""The status word of packed attention's default workspace."""
import pytest
import torch

from paper_2607_20507_gb300 import binding

pytestmark = pytest.mark.gpu

DEV = "cuda:0"


@pytest.mark.parametrize("G", [4, 8])      # 20 and 40 query rows: one form, and the other
def test_default_workspace_and_its_status(G):
    H, ps, k = 2, 16, 4
    pool = binding.packed_pool(8, H, ps, DEV)
    q = torch.randn(2, k + 1, H * G, 128, generator=torch.Generator().manual_seed(0)).bfloat16().to(DEV)
    table = torch.arange(8, dtype=torch.int32, device=DEV).view(2, 4)
    lens = torch.tensor([64, 33], dtype=torch.int32, device=DEV)
    dims = binding.packed_attn_dims(q, pool, table)
    side = torch.cuda.Stream()
    seen = []
    for stream in (torch.cuda.current_stream(), side):
        with torch.cuda.stream(stream):
            binding.cs_packed_verify_attention(q, pool, table, lens, k)
            ws = binding.packed_verify_attention_workspace(dims, k, DEV)
            assert binding.cs_read_device_status(ws) == 0
            word = ws[:4].view(torch.int32)
            word.fill_(0x77)                # any contents: each call clears it, so this is its workspace
            assert binding.cs_read_device_status(ws) == 0x77
            binding.cs_packed_verify_attention(q, pool, table, lens, k)
            assert binding.cs_read_device_status(ws) == 0
            # a wait that gives up in it would show
            binding.cs_selftest_wait_timeout(ws)
            assert binding.cs_read_device_status(ws) & binding.CS_DEVICE_WAIT_TIMEOUT
            binding.cs_packed_verify_attention(q, pool, table, lens, k)
            assert binding.cs_read_device_status(ws) == 0
            assert binding.packed_verify_attention_workspace(dims, k, DEV, stream.cuda_stream).data_ptr() == ws.data_ptr()
            seen.append(ws.data_ptr())
    assert seen[0] != seen[1]
