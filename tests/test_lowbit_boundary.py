"""CPU-side checks of the low-bit serving operators: arguments are refused on the host before anything is launched, sizes of
pages and workspaces, and the reference of the GPU tests against closed forms (no GPU needed)."""
import ctypes

import numpy as np
import pytest
import torch

import lowbit_ref as ref
from paper_2509_05576_b200 import build as ptq_build

ODD = ctypes.c_void_p((1 << 46) + 4)


def at(i):
    """An address that is never dereferenced (argument checks come first), far from the others."""
    return ctypes.c_void_p(i << 40)


FAKE = at(1)


@pytest.fixture(scope="module")
def ptq():
    ptq_build.build()
    from paper_2509_05576_b200 import ptq as module
    return module


def test_reference_rounds_as_the_format_does():
    g = torch.Generator().manual_seed(1)
    x = torch.randn(4096, generator=g) * torch.exp2(torch.randint(-12, 8, (4096,), generator=g).float())
    x = x.clamp(-448, 448)
    assert np.array_equal(ref.e4m3(x.double().numpy()), x.to(torch.float8_e4m3fn).double().numpy())
    # a power-of-two scale leaves the block's largest magnitude in (224, 448]
    q, s = ref.f8_cast(x.view(8, 512).numpy(), 1)
    top = np.abs(x.view(8, 4, 128).numpy()).max(-1) / s
    assert (top <= 448).all() and (top > 224).all()


def test_reference_grid_holds_zero_and_its_values_are_half_precision_numbers():
    rng = np.random.default_rng(2)
    x = rng.standard_normal((64, 128)) * np.exp2(rng.integers(-18, 9, (64, 1)))
    x[0] = 0.0
    x[1] = np.abs(x[1])
    x[2] = -np.abs(x[2])
    c, s, z = ref.grid4(x)
    held = ref.held4(x)
    assert c.min() >= 0 and c.max() <= 15 and np.array_equal(held.astype(np.float16).astype(np.float64), held)
    assert (ref.held4(np.where(np.arange(128) % 2, x, 0.0))[:, ::2] == 0).all()          # 0 is held as 0
    step = np.repeat(s, 32, -1)
    # rounding twice (the value and the zero code) is at most a step at the ends of the range, half a step in it
    assert (np.abs(held - x) <= step * (1 + 1e-12)).all()
    assert (np.asarray(s, np.float16).view(np.uint16) & 31 == 0).all()


def test_page_and_workspace_sizes(ptq):
    size = ptq.lib().ptq_cache_page_bytes
    assert size(16, 1, 128) == 2304 and size(64, 8, 64) == 4 * 8 * 1152 and ref.tile_bytes(128) == 2304
    for bad in ((8, 1, 128), (48, 1, 128), (2048, 1, 128), (16, 0, 128), (16, 1, 96), (16, 1, 256), (0, 1, 64)):
        assert size(*bad) == 0
    ws = ptq.lib().ptq_cache_attention_workspace_bytes
    for bad in ((8, 3, 128, 1, 1, 1), (8, 2, 96, 1, 1, 1), (8, 2, 128, -1, 1, 1), (0, 1, 128, 1, 1, 1), (8, 2, 128, 1, 1 << 30, 1)):
        assert ws(*bad) == 0
    # more rows, requests or tokens never need less, and lengths do not enter
    for need in ([ws(32, 8, 128, 4, 4 * q, q) for q in (1, 2, 4, 5, 64, 100000)], [ws(32, 8, 64, 100, t, 50) for t in (1, 50, 5000)],
                 [ws(32, 8, 64, b, 5000, 50) for b in (1, 100, 10000)]):
        assert need == sorted(need) and 0 < need[0] and need[-1] < 128 << 20
    with pytest.raises(ptq.PtqError) as e:
        ptq.Cache4(4, 48, 8, 128)
    assert e.value.code == ptq.ERR_UNSUPPORTED


def test_cast_refuses_bad_arguments(ptq):
    f = ptq.lib().ptq_fp8_quantize
    ok = dict(x=at(1), x_type=ptq.BF16, rows=4, cols=200, ldx=200, block_rows=1, q=at(2), ldq=208, scale=at(3), ld_scale=2, status=at(4), stream=None)

    def call(**kw):
        return f(*{**ok, **kw}.values())

    for kw in (dict(x=None), dict(q=None), dict(scale=None), dict(rows=-1), dict(cols=0), dict(ldx=199), dict(ldq=192), dict(ld_scale=1),
               dict(x_type=3), dict(x_type=-1), dict(block_rows=64), dict(block_rows=0), dict(q=at(1)), dict(scale=at(1)), dict(scale=at(2))):
        assert call(**kw) == ptq.ERR_INVALID_ARG, kw
    assert call(ldq=200) == ptq.ERR_ALIGNMENT and call(q=ODD) == ptq.ERR_ALIGNMENT
    assert call(rows=0, x=None, q=None, scale=None) == ptq.OK


def test_product_refuses_bad_arguments(ptq):
    f = ptq.lib().ptq_fp8_matmul
    ok = dict(C=at(1), c_type=ptq.F32, ldc=100, A=at(2), lda=208, sa=at(3), ldsa=2, B=at(4), ldb=208, sb=at(5), ldsb=2, m=4, n=100, k=200,
              status=at(6), stream=None)

    def call(**kw):
        return f(*{**ok, **kw}.values())

    for kw in (dict(C=None), dict(A=None), dict(B=None), dict(sa=None), dict(sb=None), dict(m=-1), dict(n=-1), dict(k=0), dict(ldc=99),
               dict(lda=192), dict(ldb=192), dict(ldsa=1), dict(ldsb=1), dict(c_type=7), dict(C=at(2)), dict(C=at(3)), dict(C=at(4)), dict(C=at(5))):
        assert call(**kw) == ptq.ERR_INVALID_ARG, kw
    for kw in (dict(A=ODD), dict(B=ODD), dict(lda=200), dict(ldb=201)):
        assert call(**kw) == ptq.ERR_ALIGNMENT, kw
    assert call(m=(1 << 20) + 1) == ptq.ERR_UNSUPPORTED and call(n=(1 << 22) + 1, ldc=1 << 23) == ptq.ERR_UNSUPPORTED
    assert call(m=0, C=None, A=None) == ptq.OK and call(n=0) == ptq.OK


def test_plan_refuses_bad_arguments(ptq):
    f = ptq.lib().ptq_cache_plan
    ok = dict(lens=at(1), new=at(2), batch=4, page=16, table=at(3), ldt=8, max_pages=8, free=at(4), num_free=4, slots=at(5), positions=at(6),
              max_tokens=16, cu=at(7), lens_out=at(8), taken=at(9), status=at(10), stream=None)

    def call(**kw):
        return f(*{**ok, **kw}.values())

    for kw in (dict(lens=None), dict(new=None), dict(table=None), dict(free=None), dict(slots=None), dict(positions=None), dict(cu=None),
               dict(lens_out=None), dict(taken=None), dict(batch=-1), dict(ldt=7), dict(max_pages=-1), dict(num_free=-1), dict(max_tokens=-1),
               dict(lens_out=at(1)), dict(lens_out=ctypes.c_void_p((1 << 40) + 12))):
        assert call(**kw) == ptq.ERR_INVALID_ARG, kw
    outs, ins = ["table", "slots", "positions", "cu", "lens_out", "taken"], ["lens", "new", "free"]
    for i, name in enumerate(outs):                     # every output lies apart from the inputs and the other outputs
        for other in ins + outs[:i]:
            assert call(**{name: ok[other]}) == ptq.ERR_INVALID_ARG, (name, other)
    for kw in (dict(page=8), dict(page=24), dict(page=2048), dict(max_pages=1 << 28, ldt=1 << 28), dict(max_pages=(1 << 26) + 1, ldt=1 << 27)):
        assert call(**kw) == ptq.ERR_UNSUPPORTED, kw


@pytest.mark.parametrize("name", ["ptq_cache_append", "ptq_cache_read"])
def test_append_and_read_refuse_bad_arguments(ptq, name):
    f = getattr(ptq.lib(), name)
    ok = dict(pages=at(1), num_pages=4, page=16, heads=2, dim=64, k=at(2), kt=128, kh=64, v=at(3), vt=128, vh=64, type=ptq.F16, slots=at(4),
              tokens=3, status=at(5), stream=None)

    def call(**kw):
        return f(*{**ok, **kw}.values())

    for kw in (dict(pages=None), dict(num_pages=0), dict(heads=0), dict(dim=0), dict(k=None), dict(v=None), dict(slots=None), dict(type=9),
               dict(tokens=-1), dict(kt=-1)):
        assert call(**kw) == ptq.ERR_INVALID_ARG, kw
    for kw in (dict(page=17), dict(dim=80), dict(dim=256), dict(num_pages=1 << 28), dict(heads=70000)):
        assert call(**kw) == ptq.ERR_UNSUPPORTED, kw
    assert call(pages=ODD) == ptq.ERR_ALIGNMENT
    assert call(tokens=0, k=None, v=None, slots=None) == ptq.OK
    if name == "ptq_cache_read":                       # rows that overlap cannot be written
        assert call(kt=32) == ptq.ERR_INVALID_ARG and call(vh=0) == ptq.ERR_INVALID_ARG
        assert call(k=at(1)) == ptq.ERR_INVALID_ARG and call(v=at(4)) == ptq.ERR_INVALID_ARG


def test_attention_refuses_bad_arguments(ptq):
    f = ptq.lib().ptq_cache_attention
    ok = dict(out=at(1), ot=512, oh=64, lse=at(2), q=at(3), qt=512, qh=64, type=ptq.BF16, q_heads=8, pages=at(4), num_pages=4, page=16, heads=2,
              dim=64, table=at(5), ldt=8, max_pages=8, lens=at(6), cu=at(7), batch=2, total=2, max_q=1, scale=0.125, causal=1, window=0,
              ws=at(8), ws_bytes=1 << 30, status=at(9), stream=None)

    def call(**kw):
        return f(*{**ok, **kw}.values())

    for kw in (dict(out=None), dict(q=None), dict(pages=None), dict(table=None), dict(lens=None), dict(cu=None), dict(type=ptq.F32), dict(type=5),
               dict(q_heads=7), dict(q_heads=0), dict(ldt=7), dict(batch=-1), dict(total=-1), dict(max_q=-1), dict(window=-1), dict(causal=2),
               dict(scale=float("nan")), dict(scale=float("inf")), dict(ot=32), dict(oh=0), dict(qt=-1)):
        assert call(**kw) == ptq.ERR_INVALID_ARG, kw
    names = ["out", "lse", "ws", "q", "pages", "table", "lens", "cu"]
    for i, name in enumerate(names[:3]):
        for other in names[i + 1:]:
            assert call(**{name: ok[other]}) == ptq.ERR_INVALID_ARG, (name, other)
    for kw in (dict(page=24), dict(dim=96), dict(max_pages=1 << 28, ldt=1 << 28), dict(total=1 << 30)):
        assert call(**kw) == ptq.ERR_UNSUPPORTED, kw
    assert call(pages=ODD) == ptq.ERR_ALIGNMENT and call(ws=ODD) == ptq.ERR_ALIGNMENT
    assert call(ws=None) == ptq.ERR_WORKSPACE and call(ws_bytes=64) == ptq.ERR_WORKSPACE
    for kw in (dict(batch=0), dict(total=0), dict(max_q=0)):
        assert call(**kw) == ptq.OK, kw


def test_binding_refuses_what_the_library_cannot_see(ptq):
    x = torch.zeros(4, 128)
    with pytest.raises(ValueError):                     # no CPU path
        ptq.fp8_quantize(x, torch.zeros(4, 128, dtype=torch.uint8), torch.zeros(4, 1), torch.zeros(4, dtype=torch.int32))
    with pytest.raises(ValueError):
        ptq.fp8_matmul(x, x, x, x, x, None)
    with pytest.raises(ValueError):
        ptq.Cache4(2, 16, 1, 64, pages=torch.zeros(2, 1, 1, 1152, dtype=torch.uint8))
    assert ptq.fp8_empty(3, 100, device="cpu").stride() == (112, 1)
