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


def _meet(first, second, tokens, heads, by_token, by_head, dim):
    """Whether two sets of rows of elements share one: brute force."""
    a = {first + i * by_token + j * by_head + e for i in range(tokens) for j in range(heads) for e in range(dim)}
    b = {second + i * by_token + j * by_head + e for i in range(tokens) for j in range(heads) for e in range(dim)}
    return bool(a & b)


def test_read_writes_keys_and_values_apart(ptq):
    """k and v of one shape anywhere in one buffer: refused where they share an element.  (Where they do not, the call would be
    launched: those are GPU tests.)"""
    ok, f = _tokens(ptq), ptq.lib().ptq_cache_read
    for by_token, by_head in ((128, 64), (256, 64), (256, 128), (64, 192), (70, 300), (300, 70)):
        for shift in (0, 1, 63, 64, 65, 69, 70, 100, 127, 128, 130, 191, 192, 193, 255, 256, 330, 384, 600, 700):
            for sign in (1, -1):
                if _meet(0, sign * shift, 3, 2, by_token, by_head, 64):
                    kw = dict(kt=by_token, kh=by_head, vt=by_token, vh=by_head, v=at(2, sign * shift * 2))
                    assert _call(f, ok, **kw) == ptq.ERR_INVALID_ARG, (by_token, by_head, shift * sign)
    assert _call(f, ok, v=at(2, 64 * 2), vt=256) == ptq.ERR_INVALID_ARG             # other strides: all bytes between
    for kw in (dict(kt=64), dict(kh=128), dict(kt=100, kh=100), dict(vt=64), dict(vh=256)):              # rows of one output overlap
        assert _call(f, ok, **kw) == ptq.ERR_INVALID_ARG, kw


def test_attention_writes_rows_apart(ptq):
    f = ptq.lib().ptq_cache_attention
    ok = dict(out=at(1), ot=512, oh=64, lse=at(2), q=at(3), qt=512, qh=64, type=ptq.BF16, q_heads=8, pages=at(4), num_pages=4, page=16, heads=2,
              dim=64, table=at(5), ldt=8, max_pages=8, lens=at(6), cu=at(7), batch=2, total=2, max_q=1, scale=0.125, causal=1, window=0,
              ws=at(8), ws_bytes=1 << 30, status=at(9), stream=None)
    for kw in (dict(ot=64), dict(ot=448), dict(oh=512), dict(ot=100, oh=100), dict(out=at(3)), dict(out=at(3, 64 * 2)), dict(out=at(3, -1000)),
               dict(out=at(3, 1024), ot=600), dict(out=at(3, 510), qt=2048, ot=2048)):
        assert _call(f, ok, **kw) == ptq.ERR_INVALID_ARG, kw
