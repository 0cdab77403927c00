"""The low-bit serving operators on the GPU against their definitions in 64 bits (``lowbit_ref``).

Tolerances.  A cast and a slot are exact.  Sums on the tensor cores and in registers are float32: n products sum to within
n 2^-23 of the sum of their magnitudes, whatever the order (each addition is off by at most one unit in the last place, 2^-23,
of a partial sum, which the sum of magnitudes bounds).  The rounding to the output type is half a step of it.
Attention: a score is off by at most d = (dim + 4) 2^-23 max |q| |k| |scale| (the sum, the factor and their product), and the
exponential by 2^-22 relative (ex2.approx is good to 2 units in the last place); a probability is then off by e = 2 d + 2^-21
relative (numerator and sum), enters the second product rounded to fp16 (2^-11 relative; below the normal range half a step is
2^-25, where the largest probability stands at 2^8 or more: 2^-33 of it) and the output is off by (e + 2^-11 + n 2^-23) sum p |v|
plus n 2^-33 max |v| plus the rounding of the type.
"""
import numpy as np
import pytest
import torch

import lowbit_ref as ref
from paper_2509_05576_b200 import ptq

pytestmark = pytest.mark.gpu
HALF_STEP = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
TINY = {torch.float32: 2.0 ** -149, torch.float16: 2.0 ** -25, torch.bfloat16: 2.0 ** -134}


def _gen(seed):
    return torch.Generator().manual_seed(seed)


def _cast(x, rows, status):
    q = ptq.fp8_empty(*x.shape)
    s = torch.empty(-(-x.shape[0] // rows), -(-x.shape[1] // 128), device="cuda")
    ptq.fp8_quantize(x, q, s, status, block_rows=rows)
    return q, s


# ---------------------------------------------------------------------------------------------------------------- cast
@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16])
@pytest.mark.parametrize("rows", [1, 128])
@pytest.mark.parametrize("shape", [(1, 1), (1, 128), (3, 129), (128, 256), (130, 1000), (257, 131), (64, 4096)])
def test_cast_is_exact(shape, rows, dtype):
    g = _gen(sum(shape) + rows)
    x = torch.randn(shape, generator=g) * torch.exp2(torch.randint(-8, 8, (1, shape[1]), generator=g).float())
    x[0, 0] = 0.0
    if shape[0] > 2:
        x[2] = 0.0                                               # an empty row or part of a block
    x = x.to(dtype)
    st = ptq.new_status()
    q, s = _cast(x.cuda(), rows, st)
    ptq.check_status(st)
    rq, rs = ref.f8_cast(x.double().numpy(), rows)
    assert np.array_equal(s.cpu().double().numpy(), rs)
    assert np.array_equal(q.cpu().double().numpy(), rq)


def test_cast_at_the_ends_of_the_range():
    # magnitudes at and next to 448 2^e, subnormal inputs, the largest number, a block of equal values
    rows = []
    for top in (448.0, np.nextafter(np.float32(448), np.float32(449)), 1.0, 0.875, 3.0e38, 1e-38, 1e-42, 2.0 ** -130):
        r = np.linspace(-1, 1, 128).astype(np.float32) * np.float32(top)
        r[5] = top
        rows.append(r)
    x = torch.from_numpy(np.stack(rows))
    st = ptq.new_status()
    q, s = _cast(x.cuda(), 1, st)
    ptq.check_status(st)
    rq, rs = ref.f8_cast(x.double().numpy(), 1)
    assert np.array_equal(s.cpu().double().numpy(), rs) and np.array_equal(q.cpu().double().numpy(), rq)


@pytest.mark.parametrize("rows", [1, 128])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_cast_reports_what_is_not_finite(rows, bad):
    x = torch.randn(140, 300, generator=_gen(3))
    x[130, 200] = bad
    st = ptq.new_status()
    q, s = _cast(x.cuda(), rows, st)
    with pytest.raises(ptq.PtqError) as e:
        ptq.check_status(st)
    assert e.value.code == ptq.ERR_NONFINITE and e.value.index == (130 if rows == 1 else 128)
    hit = torch.zeros(140, 300, dtype=torch.bool)
    hit[130 if rows == 1 else slice(128, 140), 128:256] = True
    assert torch.equal(torch.isnan(q.cpu().float()), hit)
    assert torch.isnan(s.cpu()).sum() == 1


def test_cast_takes_any_stride_and_leaves_the_rest():
    x = torch.randn(37, 515, generator=_gen(4)).cuda()
    view = x[:, 1:301]                                           # rows that do not begin on 16 bytes
    buf = torch.full((37, 320), 77, dtype=torch.uint8, device="cuda")
    sbuf = torch.full((37, 9), -1.0, device="cuda")
    st = ptq.new_status()
    ptq.fp8_quantize(view, buf[:, :300], sbuf[:, :3], st)
    ptq.check_status(st)
    rq, rs = ref.f8_cast(view.cpu().double().numpy(), 1)
    assert np.array_equal(buf[:, :300].contiguous().view(torch.float8_e4m3fn).cpu().double().numpy(), rq)
    assert np.array_equal(sbuf[:, :3].cpu().double().numpy(), rs)
    assert (buf[:, 300:] == 77).all() and (sbuf[:, 3:] == -1).all()


# ------------------------------------------------------------------------------------------------------------- product
def _operands(m, n, k, seed, power=True):
    g = _gen(seed)
    st = ptq.new_status()
    a = torch.randn(m, k, generator=g) * torch.exp2(torch.randint(-4, 4, (1, k), generator=g).float())
    b = torch.randn(n, k, generator=g) / k ** 0.5
    A, sa = _cast(a.cuda(), 1, st)
    B, sb = _cast(b.cuda(), 128, st)
    if not power:                                                # any float32 scales are taken
        sa = sa * (torch.rand(sa.shape, generator=g) + 0.5).cuda()
        sb = sb * (torch.rand(sb.shape, generator=g) + 0.5).cuda()
    ptq.check_status(st)
    return A, sa, B, sb


def _check_product(C, A, sa, B, sb):
    a = ref.f8_values(A.cpu().double().numpy(), sa.cpu().double().numpy(), 1)
    b = ref.f8_values(B.cpu().double().numpy(), sb.cpu().double().numpy(), 128)
    want, mass = a @ b.T, np.abs(a) @ np.abs(b).T
    kb = sa.shape[1]
    # 128 products a block, a factor and an addition a block, the sums of up to eight CTAs, the rounding
    tol = (128 + 2 * kb + 8) * 2.0 ** -23 * mass + HALF_STEP[C.dtype] * np.abs(want) + TINY[C.dtype]
    off = np.abs(C.cpu().double().numpy() - want)
    assert (off <= tol).all(), (off - tol).max()


PRODUCTS = [(1, 1, 1), (1, 128, 128), (1, 1000, 2048), (1, 4096, 1024), (2, 130, 129), (15, 256, 384), (16, 64, 4096), (17, 300, 500), (33, 129, 700),
            (64, 512, 2304), (65, 257, 1000), (128, 256, 128), (200, 1000, 1000), (333, 1000, 2048), (1, 256, 11008), (5, 384, 2200), (3, 20000, 256),
            (66, 9000, 200)]


@pytest.mark.parametrize("m,n,k", PRODUCTS)
def test_product(m, n, k):
    A, sa, B, sb = _operands(m, n, k, m + n + k, power=k % 2 == 0)
    C = torch.full((m, n), float("nan"), device="cuda")
    st = ptq.new_status()
    ptq.fp8_matmul(C, A, sa, B, sb, st)
    ptq.check_status(st)
    _check_product(C, A, sa, B, sb)


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16])
@pytest.mark.parametrize("m,n,k", [(2100, 2500, 300), (4000, 1300, 129), (9, 700, 260)])
def test_product_of_many_rows_and_each_type(m, n, k, dtype):
    A, sa, B, sb = _operands(m, n, k, 5)
    C = torch.full((m, n), float("nan"), dtype=dtype, device="cuda")
    st = ptq.new_status()
    ptq.fp8_matmul(C, A, sa, B, sb, st)
    ptq.check_status(st)
    _check_product(C, A, sa, B, sb)


@pytest.mark.parametrize("m,n", [(7, 300), (2100, 2300)])
def test_product_strides_and_what_lies_beside(m, n):
    k = 200
    A, sa, B, sb = _operands(m, n, k, 6)
    bigA = torch.full((m, 256), 0x7F, dtype=torch.uint8, device="cuda")          # NaN codes behind the rows are not read
    bigA[:, :k] = A.view(torch.uint8)
    bigB = torch.full((n, 304), 0x7F, dtype=torch.uint8, device="cuda")
    bigB[:, :k] = B.view(torch.uint8)
    wide_a = torch.full((m, 5), float("nan"), device="cuda")
    wide_a[:, :2] = sa
    C = torch.full((m + 2, n + 3), 7.0, dtype=torch.bfloat16, device="cuda")
    st = ptq.new_status()
    ptq.fp8_matmul(C[1:m + 1, 1:n + 1], bigA[:, :k].view(torch.float8_e4m3fn), wide_a[:, :2], bigB[:, :k], sb, st)
    ptq.check_status(st)
    _check_product(C[1:m + 1, 1:n + 1], A, sa, B, sb)
    C[1:m + 1, 1:n + 1] = 7.0
    assert (C == 7.0).all()


@pytest.mark.parametrize("m", [3, 2100])
def test_what_is_not_finite_stays_in_its_row(m):
    x = torch.randn(m, 300, generator=_gen(7))
    x[1, 7] = float("inf")
    st = ptq.new_status()
    A, sa = _cast(x.cuda(), 1, st)
    _, _, B, sb = _operands(1, 2300, 300, 8)
    C = torch.empty(m, 2300, device="cuda")
    ptq.fp8_matmul(C, A, sa, B, sb, st)
    assert torch.isnan(C[1]).all() and torch.isfinite(C[0]).all() and torch.isfinite(C[2:]).all()


def test_product_gives_the_same_bits_again_and_on_another_stream():
    for m, n, k in ((1, 4096, 2048), (100, 700, 900), (2100, 2300, 400)):
        A, sa, B, sb = _operands(m, n, k, 9)
        outs = [torch.empty(m, n, device="cuda") for _ in range(3)]
        st = ptq.new_status()
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        ptq.fp8_matmul(outs[0], A, sa, B, sb, st)
        ptq.fp8_matmul(outs[1], A, sa, B, sb, st)
        ptq.fp8_matmul(outs[2], A, sa, B, sb, st, stream=side)
        torch.cuda.synchronize()
        assert torch.equal(outs[0], outs[1]) and torch.equal(outs[0], outs[2])


# ---------------------------------------------------------------------------------------------------------------- plan
class Batch:
    """Requests with cached and new tokens, their tables and a cache that holds the cached ones."""

    def __init__(self, lens, new, page, seed=0, spare=3, pad=0, width=None):
        rng = np.random.default_rng(seed)
        self.lens, self.new, self.page = list(lens), list(new), page
        have = [-(-x // page) for x in lens]
        want = [-(-(x + y) // page) for x, y in zip(lens, new)]
        self.num_pages = sum(want) + spare
        order = rng.permutation(self.num_pages).astype(np.int32)
        self.table = np.full((len(lens), width or max(want + [0]) + 1), -1, np.int32)
        at = 0
        for b, h in enumerate(have):
            self.table[b, :h] = order[at:at + h]
            at += h
        self.free = order[at:]
        self.tokens = sum(new) + pad

    def plan(self, status=None):
        st = status if status is not None else ptq.new_status()
        c = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
        self.d_table, self.d_lens, self.d_new, self.d_free = c(self.table), c(self.lens), c(self.new), c(self.free)
        e = lambda n: torch.full((n,), 12345, dtype=torch.int32, device="cuda")  # noqa: E731
        self.slots, self.positions, self.cu, self.lens_out, self.taken = (e(self.tokens), e(self.tokens), e(len(self.lens) + 1),
                                                                           e(len(self.lens)), e(1))
        ptq.cache_plan(self.d_lens, self.d_new, self.d_table, self.d_free, self.page, self.slots, self.positions, self.cu, self.lens_out,
                       self.taken, st)
        return st


BATCHES = [([0], [1], 16), ([15], [1], 16), ([16], [1], 16), ([5, 0, 31, 64], [1, 0, 2, 33], 16), ([1000] * 70, [1] * 70, 32), ([0] * 3, [0] * 3, 16),
           ([7, 0, 300], [5000, 1, 9000], 64), (list(range(0, 2600)), [i % 3 for i in range(2600)], 16), ([100] * 1500, [1] * 1500, 128), ([], [], 16)]


@pytest.mark.parametrize("lens,new,page", BATCHES)
@pytest.mark.parametrize("pad", [0, 5000])
def test_plan(lens, new, page, pad):
    b = Batch(lens, new, page, pad=pad, width=None if lens else 4)
    st = b.plan()
    ptq.check_status(st)
    table, slots, positions, cu, after, taken = ref.plan(lens, new, b.table, b.free, page)
    assert np.array_equal(b.d_table.cpu().numpy(), table)
    assert b.slots.tolist() == slots + [-1] * pad and b.positions.tolist() == positions + [-1] * pad
    assert b.cu.tolist() == cu and b.lens_out.tolist() == after and b.taken.tolist() == [taken]
    assert len(set(slots)) == len(slots)


@pytest.mark.parametrize("kind", ["pages", "table", "tokens", "negative", "new"])
@pytest.mark.parametrize("count", [3, 1400])
def test_plan_that_does_not_fit_does_nothing(kind, count):
    b = Batch([20] * count, [30] * count, 16)
    if kind == "pages":
        b.free = b.free[:2 * count - 1]
    elif kind == "table":
        b.table = b.table[:, :3].copy()
    elif kind == "tokens":
        b.tokens -= 1
    elif kind == "negative":
        b.lens[count - 1] = -1
    else:
        b.new[count - 1] = -2
    st = b.plan()
    with pytest.raises(ptq.PtqError) as e:
        ptq.check_status(st)
    assert e.value.code == ptq.ERR_INVALID_ARG and e.value.index == (0 if kind == "table" else count - 1)
    assert np.array_equal(b.d_table.cpu().numpy(), b.table) and b.lens_out.tolist() == b.lens
    assert (b.slots == -1).all() and (b.positions == -1).all() and (b.cu == 0).all() and b.taken.tolist() == [0]


def test_plan_records_page_numbers_that_are_none():
    b = Batch([20, 20], [5, 5], 16)
    b.table[1, 1] = -7
    st = b.plan()
    with pytest.raises(ptq.PtqError) as e:
        ptq.check_status(st)
    assert e.value.code == ptq.ERR_INVALID_ARG and e.value.index == 1
    assert (b.slots[5:] == -1).all() and (b.slots[:5] >= 0).all()


# ------------------------------------------------------------------------------------------------------- append and read
@pytest.mark.parametrize("dtype", [torch.float32, torch.float16, torch.bfloat16])
@pytest.mark.parametrize("dim,heads,page", [(64, 1, 16), (64, 3, 64), (128, 8, 32), (128, 1, 1024)])
def test_append_then_read(dim, heads, page, dtype):
    g = _gen(dim + heads)
    tokens, num_pages = 45, -(-100 // page) + 1
    k = (torch.randn(tokens, heads, dim, generator=g) * torch.exp2(torch.randint(-6, 7, (tokens, 1, 1), generator=g).float())).to(dtype)
    v = torch.randn(tokens, heads, dim, generator=g).to(dtype)
    k[3] = 0
    v[4] = v[4].abs()
    k[5] = -k[5].abs()
    cache = ptq.Cache4(num_pages, page, heads, dim)
    cache.pages.fill_(0xA5)
    slots = torch.randperm(num_pages * page, generator=g)[:tokens].to(torch.int32)
    slots[7] = -1
    st = ptq.new_status()
    ptq.cache_append(cache, k.cuda(), v.cuda(), slots.cuda(), st)
    out = [torch.full((tokens, heads, dim), 9.0, dtype=dtype, device="cuda") for _ in range(2)]
    ptq.cache_read(cache, slots.cuda(), *out, st)
    ptq.check_status(st)
    keep = slots >= 0
    for got, x in zip(out, (k, v)):
        held = ref.held4(x.double().numpy())
        want = torch.from_numpy(held).to(dtype)                   # bf16 has fewer bits than what is held
        assert torch.equal(got.cpu()[keep], want[keep]) and (got[~keep] == 9.0).all()
    # the bytes themselves, and nothing but the written slots
    blank = cache.pages.cpu().numpy()
    kk, vv = np.zeros((num_pages, heads, page, dim)), np.zeros((num_pages, heads, page, dim))
    for i, s in enumerate(slots.tolist()):
        if s >= 0:
            kk[s // page, :, s % page], vv[s // page, :, s % page] = k[i].double().numpy(), v[i].double().numpy()
    full = ref.pages_from(kk, vv)
    written = np.zeros((num_pages, page), bool)
    written.reshape(-1)[slots[keep].numpy()] = True
    side, codes = ref.tile_bytes(dim) // 2, 16 * dim // 2
    for p in range(num_pages):
        for r in range(page):
            for base in (0, side):
                for lo, hi in ((base + r % 16 * dim // 2, base + (r % 16 + 1) * dim // 2),
                               (base + codes + r % 16 * dim // 16, base + codes + (r % 16 + 1) * dim // 16)):
                    got = blank[p, :, r // 16, lo:hi]
                    assert (got == (full[p, :, r // 16, lo:hi] if written[p, r] else 0xA5)).all()


def test_append_takes_strided_tokens_and_heads():
    g = _gen(11)
    packed = torch.randn(20, 3, 2, 4, 128, generator=g).to(torch.bfloat16).cuda()          # q, k, v of a fused projection
    k, v = packed[:, 1, 0], packed[:, 2, 1]
    odd = torch.randn(20, 4 * 128 + 3, generator=g).to(torch.bfloat16).cuda()[:, 3:].unflatten(1, (4, 128))
    for kk, vv in ((k, v), (odd, v)):
        cache = ptq.Cache4(2, 16, 4, 128)
        slots = torch.arange(20, dtype=torch.int32, device="cuda")
        st = ptq.new_status()
        ptq.cache_append(cache, kk, vv, slots, st)
        out = [torch.empty(4, 20, 128, device="cuda").transpose(0, 1) for _ in range(2)]
        ptq.cache_read(cache, slots, *out, st)
        ptq.check_status(st)
        for got, x in zip(out, (kk, vv)):
            assert np.array_equal(got.cpu().double().numpy(), ref.held4(x.cpu().double().numpy()))


def test_append_at_the_ends_of_the_range():
    dim = 64
    tops = [1e-12, 2.0 ** -19, 1e-4, 6e4, 3e38]
    x = torch.zeros(len(tops), 1, dim)
    for i, t in enumerate(tops):
        x[i, 0] = torch.linspace(-1, 1, dim) * t
    cache = ptq.Cache4(1, 16, 1, dim)
    slots = torch.arange(len(tops), dtype=torch.int32, device="cuda")
    st = ptq.new_status()
    ptq.cache_append(cache, x.cuda(), x.cuda(), slots, st)
    k, v = torch.empty(len(tops), 1, dim, device="cuda"), torch.empty(len(tops), 1, dim, device="cuda")
    ptq.cache_read(cache, slots, k, v, st)
    ptq.check_status(st)
    assert np.array_equal(k.cpu().double().numpy(), ref.held4(x.double().numpy())) and torch.equal(k, v)
    assert float(k.abs().max()) <= 15 * 2112


def test_append_keeps_the_cache_finite_and_says_so():
    x = torch.randn(5, 2, 128, generator=_gen(12))
    x[2, 1, 40] = float("nan")
    x[2, 0, 3] = float("inf")
    x[2, 0, 70] = -float("inf")
    cache = ptq.Cache4(1, 16, 2, 128)
    cache.pages.zero_()
    slots = torch.arange(5, dtype=torch.int32, device="cuda")
    st = ptq.new_status()
    ptq.cache_append(cache, x.cuda(), x.cuda(), slots, st)
    with pytest.raises(ptq.PtqError) as e:
        ptq.check_status(st)
    assert e.value.code == ptq.ERR_NONFINITE and e.value.index == 2
    k, v = torch.empty(5, 2, 128, device="cuda"), torch.empty(5, 2, 128, device="cuda")
    ptq.cache_read(cache, slots, k, v, ptq.new_status())
    assert torch.isfinite(k).all() and float(k[2, 1, 40]) == 0.0
    assert float(k[2, 0, 3]) == 15 * 2112 and float(k[2, 0, 70]) == -15 * 2112


def test_append_and_read_skip_slots_that_are_none():
    cache = ptq.Cache4(2, 16, 1, 64)
    cache.pages.zero_()
    before = cache.pages.clone()
    x = torch.randn(3, 1, 64, generator=_gen(13)).cuda()
    slots = torch.tensor([-1, 32, 2 ** 31 - 1], dtype=torch.int32, device="cuda")
    for call in (lambda st: ptq.cache_append(cache, x, x, slots, st), lambda st: ptq.cache_read(cache, slots, x, x.clone(), st)):
        st = ptq.new_status()
        call(st)
        with pytest.raises(ptq.PtqError) as e:
            ptq.check_status(st)
        assert e.value.code == ptq.ERR_INVALID_ARG and e.value.index in (1, 2)
    assert torch.equal(cache.pages, before)


# ----------------------------------------------------------------------------------------------------------- attention
def _attend(lens, new, heads, kv_heads, dim, page, dtype, causal=True, window=0, seed=0, scale=None, extra_rows=0, want_lse=True, garbage=True,
            q_gain=1.0, strided=False, ws=None, check=True, max_q=None):
    """Requests whose `lens` tokens are cached and the last `new` of them ask; compares with the definition."""
    rng = np.random.default_rng(seed)
    b = Batch(lens, [0] * len(lens), page, seed=seed)
    cache = ptq.Cache4(b.num_pages, page, kv_heads, dim)
    if garbage:                                                  # what no request holds may be anything, NaN among it
        cache.pages.copy_(torch.from_numpy(rng.integers(0, 256, tuple(cache.pages.shape), dtype=np.uint8)))
        cache.pages[:, :, :, 16 * dim // 2:16 * dim // 2 + 7] = 0xFF
        cache.pages[:, :, :, -9:] = 0xFF
    st = ptq.new_status()
    keys, vals = [], []
    for i, n in enumerate(lens):
        k = (rng.standard_normal((n, kv_heads, dim)) * np.exp2(rng.standard_normal((1, kv_heads, dim)))).astype(np.float32)
        v = rng.standard_normal((n, kv_heads, dim)).astype(np.float32)
        keys.append(ref.held4(k) if n else k)
        vals.append(ref.held4(v) if n else v)
        j = np.arange(n)
        slots = torch.tensor((b.table[i, j // page] * page + j % page).astype(np.int32), device="cuda")
        if n:
            ptq.cache_append(cache, torch.from_numpy(k).cuda(), torch.from_numpy(v).cuda(), slots, st)
    total = sum(new) + extra_rows
    q = torch.from_numpy(rng.standard_normal((total, heads, dim)) * q_gain).to(dtype)
    scale = dim ** -0.5 if scale is None else scale
    c = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    cu = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
    if strided:
        dq = torch.zeros(heads, total, dim + 8, dtype=dtype, device="cuda")[:, :, 3:dim + 3].transpose(0, 1)
        dq.copy_(q)
        out = torch.full((heads, total, dim + 1), 5.0, dtype=dtype, device="cuda")[:, :, :dim].transpose(0, 1)
    else:
        dq, out = q.cuda(), torch.full((total, heads, dim), 5.0, dtype=dtype, device="cuda")
    lse = torch.full((total, heads), 5.0, device="cuda") if want_lse else None
    ptq.cache_attention(out, dq, cache, c(b.table), c(lens), c(cu), max(new + [0]) if max_q is None else max_q, scale, ws or ptq.Workspace(), st,
                        causal=causal, window=window, lse=lse)
    ptq.check_status(st)
    got, got_lse = out.cpu().double().numpy(), None if lse is None else lse.cpu().double().numpy()
    if check:
        for i, (n, m) in enumerate(zip(lens, new)):
            at = slice(cu[i], cu[i + 1])
            want, want_lse_, mass, reach = ref.attention(q[at].double().numpy(), keys[i], vals[i], n, scale, causal, window)
            d = (dim + 4) * 2.0 ** -23 * reach
            e = (2 * d + 2.0 ** -21)[..., None]
            tol = (e + 2.0 ** -11 + max(n, 1) * 2.0 ** -23) * mass + HALF_STEP[dtype] * np.abs(want) + TINY[dtype]
            if n:
                tol = tol + n * 2.0 ** -33 * np.abs(vals[i]).max()
            off = np.abs(got[at] - want)
            assert (off <= tol).all(), (i, float((off - tol).max()))
            if lse is not None:
                none = np.isneginf(want_lse_)
                assert (np.isneginf(got_lse[at]) == none).all()
                off = np.abs(got_lse[at][~none] - want_lse_[~none])
                assert (off <= d[~none] + max(n, 1) * 2.0 ** -23 + 2.0 ** -21 * (2 + np.abs(want_lse_[~none]))).all(), off.max()
        assert (got[cu[-1]:] == 5.0).all() and (got_lse is None or (got_lse[cu[-1]:] == 5.0).all())
    return out, lse


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("heads,kv_heads", [(1, 1), (4, 2), (8, 1), (7, 1), (12, 1), (16, 1), (6, 2)])
def test_one_token_each(heads, kv_heads, dim, dtype):
    _attend([1, 15, 16, 17, 33, 200, 0, 513], [1] * 8, heads, kv_heads, dim, 16, dtype, seed=heads + dim)


@pytest.mark.parametrize("page", [16, 32, 128, 1024])
def test_pages(page):
    _attend([1, 31, 129, 1500], [1, 1, 1, 1], 8, 2, 128, page, torch.bfloat16, seed=page)


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("lens", [[9000], [20000, 3], [1, 4097, 0, 7000, 31]])
def test_long_requests_are_shared_by_many_blocks(lens, dim):
    _attend(lens, [1] * len(lens), 4, 1, dim, 64, torch.float16, seed=len(lens))


def test_more_requests_than_threads():
    rng = np.random.default_rng(5)
    lens = rng.integers(0, 70, 600).tolist()
    _attend(lens, [int(x) for x in rng.integers(0, 2, 600)], 4, 2, 64, 16, torch.bfloat16, seed=6)


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("window", [0, 1, 17, 100])
@pytest.mark.parametrize("dim,heads,kv_heads,new", [(64, 4, 2, [3, 1, 0, 4, 2]), (128, 4, 1, [40, 1, 0, 130, 7])])
def test_masks(dim, heads, kv_heads, new, causal, window):
    # a request with more rows than keys: its first rows see nothing when causal
    _attend([300, 1, 50, 60 if new[0] == 40 else 2, 0], new, heads, kv_heads, dim, 16, torch.bfloat16, causal=causal, window=window, seed=window)


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("dim,heads,kv_heads", [(64, 16, 2), (128, 8, 2), (128, 3, 3), (128, 40, 1), (64, 34, 2)])
def test_prompts(dim, heads, kv_heads, dtype):
    _attend([70, 129, 1, 333, 16], [70, 60, 1, 333, 16], heads, kv_heads, dim, 32, dtype, seed=dim + heads, window=0)


@pytest.mark.parametrize("new", [1, 5, 200])
def test_rows_behind_the_last_request_and_strides(new):
    for strided in (False, True):
        _attend([250, 400], [new, 1], 4, 2, 128, 16, torch.bfloat16, extra_rows=6, strided=strided, want_lse=not strided, seed=new)


@pytest.mark.parametrize("new", [1, 64])
@pytest.mark.parametrize("gain,scale", [(1e-30, 1e30), (1e30, 1e-31), (300.0, 0.5), (0.0, 1.0), (1.0, -0.3), (1.0, 0.0)])
def test_queries_and_scales_of_any_size(gain, scale, new):
    _attend([90, 64], [new, new], 4, 2, 64, 16, torch.bfloat16, q_gain=gain, scale=scale, seed=3)


def test_a_bound_on_the_rows_may_be_loose_or_tight():
    outs = [_attend([90, 300], [2, 30], 4, 2, 64, 16, torch.bfloat16, seed=4, max_q=m)[0] for m in (30, 31, 1000)]
    assert torch.equal(outs[0], outs[1]) and torch.equal(outs[0], outs[2])


def test_queries_that_are_not_finite_stay_in_their_rows():
    dim, lens = 64, [100, 100]
    for bad in (float("nan"), float("inf")):
        for new in (1, 40):
            b = Batch(lens, [0, 0], 16)
            cache = ptq.Cache4(b.num_pages, 16, 1, dim)
            x = torch.randn(200, 1, dim, generator=_gen(1)).cuda()
            c = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
            slots = c(np.concatenate([b.table[i, np.arange(100) // 16] * 16 + np.arange(100) % 16 for i in range(2)]))
            st = ptq.new_status()
            ptq.cache_append(cache, x, x, slots, st)
            q = torch.randn(2 * new, 4, dim, generator=_gen(2)).to(torch.bfloat16)
            q[0, 1, 5] = bad
            out, lse = torch.empty(2 * new, 4, dim, dtype=torch.bfloat16, device="cuda"), torch.empty(2 * new, 4, device="cuda")
            ptq.cache_attention(out, q.cuda(), cache, c(b.table), c(lens), c([0, new, 2 * new]), new, 0.125, ptq.Workspace(), st, lse=lse)
            ptq.check_status(st)
            hit = torch.zeros(2 * new, 4, dtype=torch.bool)
            hit[0, 1] = True
            assert torch.equal(~torch.isfinite(out.cpu().float()).all(-1), hit)


def test_attention_records_lengths_and_pages_that_are_none():
    b = Batch([40, 40], [0, 0], 16)
    cache = ptq.Cache4(b.num_pages, 16, 2, 64)
    cache.pages.zero_()
    q = torch.randn(2, 4, 64, generator=_gen(1)).to(torch.float16).cuda()
    c = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    wrong = b.table.copy()
    wrong[1, 2] = b.num_pages
    for table, lens, cu in ((wrong, [40, 40], [0, 1, 2]), (b.table, [40, 4000], [0, 1, 2]), (b.table, [40, -1], [0, 1, 2]), (b.table, [40, 40], [0, 1, 9])):
        st = ptq.new_status()
        out = torch.empty_like(q)
        ptq.cache_attention(out, q, cache, c(table), c(lens), c(cu), 1, 0.1, ptq.Workspace(), st)
        with pytest.raises(ptq.PtqError) as e:
            ptq.check_status(st)
        assert e.value.code == ptq.ERR_INVALID_ARG and e.value.index == 1


def test_attention_gives_the_same_bits_again_whatever_else_is_in_the_workspace():
    ws = ptq.Workspace()
    for lens, new in (([5000, 70], [1, 1]), ([3000, 700], [64, 100])):
        first = _attend(lens, new, 8, 2, 128, 64, torch.bfloat16, seed=8, ws=ws, check=False)
        ws.buf.fill_(0xFF)
        again = _attend(lens, new, 8, 2, 128, 64, torch.bfloat16, seed=8, ws=ws, check=False)
        assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])


# ------------------------------------------------------------------------------------------------------------- together
class Layer:
    """One attention layer of a low-bit network: 8-bit projections around attention over a 4-bit cache."""

    def __init__(self, requests, heads, kv_heads, dim, page, num_pages, max_pages, tokens, hidden, seed=0):
        g = _gen(seed)
        self.shape = heads, kv_heads, dim
        wide = (heads + 2 * kv_heads) * dim
        st = ptq.new_status()
        self.w_in = _cast((torch.randn(wide, hidden, generator=g) / hidden ** 0.5).cuda(), 128, st)
        self.w_out = _cast((torch.randn(hidden, heads * dim, generator=g) / (heads * dim) ** 0.5).cuda(), 128, st)
        ptq.check_status(st)
        self.cache = ptq.Cache4(num_pages, page, kv_heads, dim)
        self.page, self.status, self.ws = page, ptq.new_status(), ptq.Workspace()
        i = lambda *s: torch.zeros(s, dtype=torch.int32, device="cuda")  # noqa: E731
        self.table, self.lens, self.new, self.free = i(requests, max_pages), i(requests), i(requests), i(num_pages)
        self.slots, self.positions, self.cu, self.lens_out, self.taken = i(tokens), i(tokens), i(requests + 1), i(requests), i(1)
        self.x = torch.zeros(tokens, hidden, dtype=torch.bfloat16, device="cuda")
        self.qx, self.sx = ptq.fp8_empty(tokens, hidden), torch.empty(tokens, -(-hidden // 128), device="cuda")
        self.proj = torch.empty(tokens, wide, dtype=torch.bfloat16, device="cuda")
        self.att = torch.zeros(tokens, heads, dim, dtype=torch.bfloat16, device="cuda")
        self.qa, self.sa = ptq.fp8_empty(tokens, heads * dim), torch.empty(tokens, -(-heads * dim // 128), device="cuda")
        self.y = torch.empty(tokens, hidden, dtype=torch.bfloat16, device="cuda")

    def step(self, max_q):
        heads, kv, dim = self.shape
        st = self.status
        ptq.cache_plan(self.lens, self.new, self.table, self.free, self.page, self.slots, self.positions, self.cu, self.lens_out, self.taken, st)
        ptq.fp8_quantize(self.x, self.qx, self.sx, st)
        ptq.fp8_matmul(self.proj, self.qx, self.sx, *self.w_in, st)
        q, k, v = self.proj.unflatten(1, (-1, dim)).split([heads, kv, kv], 1)
        ptq.cache_append(self.cache, k, v, self.slots, st)
        ptq.cache_attention(self.att, q, self.cache, self.table, self.lens_out, self.cu, max_q, dim ** -0.5, self.ws, st)
        ptq.fp8_quantize(self.att.flatten(1), self.qa, self.sa, st)
        ptq.fp8_matmul(self.y, self.qa, self.sa, *self.w_out, st)


def test_a_layer_that_answers_requests_token_by_token():
    """A prompt and then single tokens of a ragged batch, all calls together, against the same in 64 bits on the values that
    the 8-bit operands and the cache hold."""
    heads, kv, dim, page, hidden = 6, 2, 64, 16, 200
    layer = Layer(3, heads, kv, dim, page, 24, 8, 64, hidden)
    layer.free.copy_(torch.randperm(24, generator=_gen(1)))
    rng = np.random.default_rng(2)
    keys, vals = [np.zeros((0, kv, dim))] * 3, [np.zeros((0, kv, dim))] * 3
    w_out = ref.f8_values(layer.w_out[0].cpu().double().numpy(), layer.w_out[1].cpu().double().numpy(), 128)
    for new in ([40, 3, 17], [1, 1, 1], [1, 0, 1], [1, 1, 1]):
        tokens = sum(new)
        layer.new.copy_(torch.tensor(new, dtype=torch.int32))
        layer.x[:tokens] = torch.from_numpy(rng.standard_normal((tokens, hidden))).to(torch.bfloat16).cuda()
        layer.step(max(new))
        ptq.check_status(layer.status)
        layer.lens.copy_(layer.lens_out)
        used = int(layer.taken)
        layer.free = layer.free[used:].contiguous()
        proj = layer.proj[:tokens].cpu().double().numpy().reshape(tokens, -1, dim)
        at = 0
        for r, n in enumerate(new):
            part = proj[at:at + n]
            if n:
                keys[r] = np.concatenate([keys[r], ref.held4(part[:, heads:heads + kv])])
                vals[r] = np.concatenate([vals[r], ref.held4(part[:, heads + kv:])])
                want, _, mass, reach = ref.attention(part[:, :heads], keys[r], vals[r], len(keys[r]), dim ** -0.5, True, 0)
                got = layer.att[at:at + n].cpu().double().numpy()
                tol = (2 * (dim + 4) * 2.0 ** -23 * reach[..., None] + 2.0 ** -10) * mass + 2.0 ** -8 * np.abs(want) + 2.0 ** -30
                assert (np.abs(got - want) <= tol).all()
            at += n
        a = ref.f8_values(*ref.f8_cast(layer.att[:tokens].cpu().double().numpy().reshape(tokens, -1), 1), 1)
        want, mass = a @ w_out.T, np.abs(a) @ np.abs(w_out).T
        assert (np.abs(layer.y[:tokens].cpu().double().numpy() - want) <= 160 * 2.0 ** -23 * mass + 2.0 ** -8 * np.abs(want) + 2.0 ** -40).all()
    assert layer.lens.tolist() == [43, 5, 20]


def test_a_captured_step_is_replayed_with_other_lengths():
    heads, kv, dim, page, hidden = 8, 2, 128, 16, 256
    layer = Layer(4, heads, kv, dim, page, 64, 16, 8, hidden, seed=1)
    layer.cache.pages.zero_()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        layer.step(1)                                            # sizes the workspace, sets kernel attributes
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        layer.step(1)
    lens = [0, 0, 0, 0]
    eager = Layer(4, heads, kv, dim, page, 64, 16, 8, hidden, seed=1)
    eager.cache.pages.zero_()
    for l in (layer, eager):
        l.table.zero_()
        l.lens.zero_()
    free = list(range(64))
    for i, new in enumerate(([1, 1, 1, 1], [1, 0, 1, 1], [0, 1, 0, 0]) + ([1, 1, 1, 1],) * 20):
        x = torch.randn(8, hidden, generator=_gen(100 + i)).to(torch.bfloat16)
        for l in (layer, eager):
            l.x.copy_(x)
            l.new.copy_(torch.tensor(new, dtype=torch.int32))
            l.lens.copy_(torch.tensor(lens, dtype=torch.int32))
            l.free.copy_(torch.tensor(free + [0] * (64 - len(free)), dtype=torch.int32))
            l.att.fill_(3.0)
        torch.cuda.synchronize()
        graph.replay()
        eager.step(1)
        torch.cuda.synchronize()
        n = sum(new)
        assert torch.equal(layer.y[:n], eager.y[:n]) and torch.equal(layer.slots, eager.slots) and torch.equal(layer.table, eager.table)
        assert (layer.att[n:] == 3.0).all() and (layer.slots[n:] == -1).all()
        free = free[int(layer.taken):]
        lens = layer.lens_out.tolist()
    for l in (layer, eager):
        ptq.check_status(l.status)
    assert lens == [22, 22, 22, 22]


def test_captured_prompts_are_replayed_with_other_lengths():
    """Single tokens and prompts in one captured batch: the launches stay, what they find on the device changes."""
    page, heads, kv, dim, batch, most, max_pages = 16, 8, 2, 64, 4, 90, 40
    cache = ptq.Cache4(batch * max_pages, page, kv, dim)
    g, st, ws = _gen(31), ptq.new_status(), ptq.Workspace()
    slots = torch.arange(batch * max_pages * page, dtype=torch.int32, device="cuda")
    kk = torch.randn(slots.numel(), kv, dim, generator=g).cuda()
    ptq.cache_append(cache, kk, kk.flip(0), slots, st)
    table = torch.randperm(batch * max_pages, generator=g).to(torch.int32).view(batch, max_pages).cuda()
    lens, cu = torch.zeros(batch, dtype=torch.int32, device="cuda"), torch.zeros(batch + 1, dtype=torch.int32, device="cuda")
    q = torch.randn(batch * most, heads, dim, generator=g).to(torch.bfloat16).cuda()
    out, lse = torch.empty_like(q), torch.empty(batch * most, heads, device="cuda")

    def step(o, l):
        ptq.cache_attention(o, q, cache, table, lens, cu, most, 0.125, ws, st, lse=l)

    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        step(out, lse)
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        step(out, lse)
    for have, new in (([90, 90, 90, 90], [90, 90, 90, 90]), ([640, 1, 300, 77], [1, 1, 80, 4]), ([5, 0, 17, 639], [5, 0, 1, 90]), ([1, 1, 1, 1], [1, 1, 1, 1]),
                      ([0, 0, 0, 0], [0, 0, 0, 0]), ([200, 640, 33, 400], [30, 2, 33, 1])):
        lens.copy_(torch.tensor(have, dtype=torch.int32))
        cu.copy_(torch.tensor([0] + list(np.cumsum(new)), dtype=torch.int32))
        out.fill_(9.0)
        lse.fill_(9.0)
        want, want_lse = out.clone(), lse.clone()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        step(want, want_lse)
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.equal(lse, want_lse)
        n = sum(new)
        assert (out[n:] == 9.0).all() and (lse[n:] == 9.0).all() and torch.isfinite(out[:n].float()).all()
    ptq.check_status(st)


def test_a_cache_beyond_32_bits_of_bytes():
    page, heads, dim = 1024, 8, 128
    num_pages = (9 << 29) // (page * heads * 144)                  # 4.5 GiB
    cache = ptq.Cache4(num_pages, page, heads, dim)
    g = _gen(5)
    k, v = torch.randn(40, heads, dim, generator=g), torch.randn(40, heads, dim, generator=g)
    slots = torch.cat([torch.arange(20), (num_pages - 1) * page + 1000 + torch.arange(20)]).to(torch.int32).cuda()
    st = ptq.new_status()
    ptq.cache_append(cache, k.cuda(), v.cuda(), slots, st)
    kb, vb = torch.empty(40, heads, dim, device="cuda"), torch.empty(40, heads, dim, device="cuda")
    ptq.cache_read(cache, slots, kb, vb, st)
    assert np.array_equal(kb.cpu().double().numpy(), ref.held4(k.double().numpy()))
    c = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    for new in (1, 20):                                            # the last page's tokens from 1000 on, reached by window
        q = torch.randn(new, 16, dim, generator=g).to(torch.float16)
        out = torch.empty(new, 16, dim, dtype=torch.float16, device="cuda")
        ptq.cache_attention(out, q.cuda(), cache, c([[num_pages - 1]]), c([1020]), c([0, new]), new, 0.1, ptq.Workspace(), st, window=1)
        want = vb[40 - new:].repeat_interleave(2, 1)               # a window of one: the row's own value, times 1 rounded to fp16 and back
        assert (out.float() - want).abs().max() <= 2.0 ** -10 * float(want.abs().max())
    ptq.check_status(st)


def test_nothing_to_do():
    st = ptq.new_status()
    e = lambda *s, t=torch.bfloat16: torch.empty(s, dtype=t, device="cuda")  # noqa: E731
    ints = lambda *s: torch.zeros(s, dtype=torch.int32, device="cuda")  # noqa: E731
    ptq.fp8_quantize(e(0, 100), ptq.fp8_empty(0, 100), e(0, 1, t=torch.float32), st)
    q, s = _cast(torch.randn(3, 128, device="cuda"), 128, st)
    ptq.fp8_matmul(e(0, 3), ptq.fp8_empty(0, 128), e(0, 1, t=torch.float32), q, s, st)
    cache, ws = ptq.Cache4(2, 16, 2, 64), ptq.Workspace()
    ptq.cache_append(cache, e(0, 2, 64), e(0, 2, 64), ints(0), st)
    ptq.cache_read(cache, ints(0), e(0, 2, 64), e(0, 2, 64), st)
    ptq.cache_attention(e(0, 4, 64), e(0, 4, 64), cache, ints(2, 3), ints(2), ints(3), 1, 0.1, ws, st)
    ptq.cache_attention(e(0, 4, 64), e(0, 4, 64), cache, ints(0, 3), ints(0), ints(1), 0, 0.1, ws, st)
    for rows in (1, 30):                                           # rows of a request that has no page at all
        out = torch.full((rows, 4, 64), 5.0, dtype=torch.bfloat16, device="cuda")
        lse = torch.full((rows, 4), 5.0, device="cuda")
        cu = torch.tensor([0, rows], dtype=torch.int32, device="cuda")
        ptq.cache_attention(out, torch.ones_like(out), cache, ints(1, 0), ints(1), cu, rows, 0.1, ws, st, lse=lse, causal=False)
        assert (out == 0).all() and torch.isneginf(lse).all()
    ptq.check_status(st)


def test_two_streams_with_workspaces_of_their_own():
    lens, new = [3000, 900, 40], [1, 20, 3]
    want = [_attend(lens, new, 8, 2, 64, 32, torch.bfloat16, seed=s, check=False) for s in (21, 22)]
    streams, got = [torch.cuda.Stream(), torch.cuda.Stream()], [None, None]
    for _ in range(3):
        for i, s in enumerate(streams):
            s.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(s):
                got[i] = _attend(lens, new, 8, 2, 64, 32, torch.bfloat16, seed=21 + i, check=False)
        torch.cuda.synchronize()
        for i in range(2):
            assert torch.equal(got[i][0], want[i][0]) and torch.equal(got[i][1], want[i][1])


def test_binding_refuses_shared_memory_and_mixed_shapes():
    st = ptq.new_status()
    x = torch.randn(4, 128, device="cuda")
    q, s = _cast(x, 1, st)
    with pytest.raises(ValueError):
        ptq.fp8_quantize(x, q, torch.empty(4, 2, device="cuda"), st)
    with pytest.raises(ValueError):
        ptq.fp8_matmul(s, q, s, q, s[:1], st)
    with pytest.raises(ptq.PtqError) as e:                       # the scales where the result would go
        ptq.fp8_matmul(s.view(torch.bfloat16)[:, :1].expand(4, 1), q, s, q[:1], s[:1], st)
    assert e.value.code == ptq.ERR_INVALID_ARG
    cache = ptq.Cache4(2, 16, 2, 64)
    t = torch.zeros(2, 2, dtype=torch.int32, device="cuda")
    qq = torch.zeros(2, 4, 64, dtype=torch.float16, device="cuda")
    args = (cache, t, t[0], torch.zeros(3, dtype=torch.int32, device="cuda"), 1, 0.1, ptq.Workspace(), st)
    with pytest.raises(ptq.PtqError) as e:
        ptq.cache_attention(qq, qq, *args)
    assert e.value.code == ptq.ERR_INVALID_ARG
    with pytest.raises(ValueError):
        ptq.cache_attention(qq.float(), qq.float() + 1, *args)
    with pytest.raises(ValueError):                              # three requests' offsets for two
        ptq.cache_attention(qq + 1, qq, cache, t, t[0], torch.zeros(4, dtype=torch.int32, device="cuda"), 1, 0.1, ptq.Workspace(), st)
    with pytest.raises(ValueError):
        ptq.cache_attention(qq + 1, qq, cache, t.cpu(), *args[2:])
