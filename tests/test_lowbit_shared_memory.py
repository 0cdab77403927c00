"""Memory that outputs of the low-bit serving calls share with inputs or with one another is refused on the host (no GPU needed:
every call here is refused before anything is launched)."""
import ctypes

import pytest

from paper_2509_05576_b200 import build as ptq_build


def at(i, offset=0):
    """An address that is never dereferenced, far from the others."""
    return ctypes.c_void_p((i << 40) + offset)


@pytest.fixture(scope="module")
def ptq():
    ptq_build.build()
    from paper_2509_05576_b200 import ptq as module
    return module


def _call(f, ok, **kw):
    return f(*{**ok, **kw}.values())


def _tokens(ptq):
    return dict(pages=at(1), num_pages=4, page=16, heads=2, dim=64, k=at(2), kt=128, kh=64, v=at(3), vt=128, vh=64, type=ptq.F16, slots=at(4), tokens=3,
                status=at(5), stream=None)


@pytest.mark.parametrize("name", ["k", "v", "slots"])
def test_append_takes_nothing_from_the_pages_it_writes(ptq, name):
    ok, f = _tokens(ptq), ptq.lib().ptq_cache_append
    size = 4 * ptq.lib().ptq_cache_page_bytes(16, 2, 64)
    for offset in (0, 16, size - 16):
        assert _call(f, ok, **{name: at(1, offset)}) == ptq.ERR_INVALID_ARG, offset
    used = 12 if name == "slots" else 2 * (2 * 128 + 64 + 64)
    assert _call(f, ok, **{name: at(1, 16 - used)}) == ptq.ERR_INVALID_ARG           # its last bytes are the first page's
    if name != "slots":                                  # a broadcast token or head, and rows that reach into the pages
        stride = dict(k=("kt", "kh"), v=("vt", "vh"))[name]
        assert _call(f, ok, **{name: at(1), stride[0]: 0, stride[1]: 0}) == ptq.ERR_INVALID_ARG
        assert _call(f, ok, **{name: at(1, -(2 << 20)), stride[0]: 1 << 20}) == ptq.ERR_INVALID_ARG
