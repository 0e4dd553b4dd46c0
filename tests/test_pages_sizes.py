"""Sizes of the page operations' workspaces (no call here reaches a kernel)."""
import ctypes

import pytest

from paper_2607_20507_gb300 import binding, build


@pytest.fixture(scope="module")
def lib():
    build.build()
    return binding.load_library()


@pytest.mark.parametrize("P", [1, 4096, 1 << 20, 2 ** 31 - 4097, 2 ** 31 - 4095, 2 ** 31 - 1])
def test_compaction_of_any_pool(lib, P):
    """Three ids a page, a count a tile of 4096 pages, and what rounding to 256 bytes adds."""
    n = lib.cs_kv_compact_workspace_bytes(ctypes.byref(binding.PageDims(4, 8, 16, P)))
    least = 256 + 12 * P + 4 * (-(-P // 4096))
    assert least <= n <= least + 4 * 256
    assert lib.cs_kv_fork_workspace_bytes(ctypes.byref(binding.PageDims(4, 8, 16, P)), 3) >= 256 + 4 * P + 24
