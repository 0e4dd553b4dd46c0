"""What the calls that carry a fork or a compaction into further pools refuse (no call here reaches a kernel)."""
import ctypes

import pytest

from paper_2607_20507_gb300 import binding, build

FAKE = 0x10000
BAD, NO_SPACE = binding.CS_ERR_INVALID_ARG, binding.CS_ERR_WORKSPACE


@pytest.fixture(scope="module")
def lib():
    build.build()
    return binding.load_library()


def page_dims(**kw):
    d = dict(rows=4, max_pages_per_seq=8, page_size=16, num_pages=100)
    d.update(kw)
    return ctypes.byref(binding.PageDims(*d.values()))


def pools(*entries):
    return (binding.PagePool * max(len(entries), 1))(*entries)


def test_more_pools_refuse(lib):
    one = pools((FAKE, 64))

    def fork(d=None, p=one, np_=1, n=2, ws=FAKE, size=1 << 40):
        return lib.cs_kv_fork_more(d or page_dims(), p, np_, n, ws, size, None)

    def compact(d=None, p=one, np_=1, ws=FAKE, size=1 << 40):
        return lib.cs_kv_compact_more(d or page_dims(), p, np_, ws, size, None)

    for call in (fork, compact):
        for name in ("rows", "max_pages_per_seq", "page_size", "num_pages"):
            assert call(page_dims(**{name: 0})) == BAD
        assert call(np_=-1) == BAD and call(np_=binding.CS_MAX_PAGE_POOLS + 1) == BAD and call(p=None) == BAD
        assert call(p=pools((None, 64))) == BAD and call(p=pools((FAKE + 8, 64))) == BAD
        assert call(p=pools((FAKE, 0))) == BAD and call(p=pools((FAKE, 24))) == BAD
        assert call(ws=None) == NO_SPACE and call(size=8) == NO_SPACE and call(ws=FAKE + 128) == BAD
        assert call(np_=0, p=None, ws=None) == binding.CS_OK
    assert fork(n=-1) == BAD and fork(n=0, ws=None) == binding.CS_OK
