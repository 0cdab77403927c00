"""Calls of the low-bit serving operators at the edges of what their documentation allows."""
import numpy as np
import pytest
import torch

import lowbit_ref as ref
import test_gpu_lowbit as base
from paper_2509_05576_b200 import ptq

pytestmark = pytest.mark.gpu


def _c(v):
    return torch.tensor(np.asarray(v, np.int32), device="cuda")


@pytest.mark.parametrize("dim,heads,kv_heads", [(64, 4, 2), (128, 8, 1)])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("new", [1, 3, 70])
@pytest.mark.parametrize("page,window", [(16, 1), (16, 40), (16, 200), (32, 130), (64, 500)])
def test_pages_below_the_window_may_be_given_back(page, window, new, causal, dim, heads, kv_heads):
    """A page whose tokens no row of the request sees any more is not read: its entry may be anything."""
    rng = np.random.default_rng(page + window)
    lens = [1000, 333, 71]
    b = base.Batch(lens, [0] * 3, page, seed=2)
    cache, st = ptq.Cache4(b.num_pages, page, kv_heads, dim), ptq.new_status()
    x = torch.from_numpy(rng.standard_normal((b.num_pages * page, kv_heads, dim)).astype(np.float32)).cuda()
    ptq.cache_append(cache, x, x.flip(0), _c(np.arange(b.num_pages * page)), st)
    q = torch.from_numpy(rng.standard_normal((3 * new, heads, dim))).to(torch.bfloat16).cuda()
    fewer, gone = b.table.copy(), 0
    for r, n in enumerate(lens):
        first = max(n - new - window + 1, 0) // page              # the page of the first row's first key
        fewer[r, :first] = [-1, b.num_pages, 2 ** 31 - 1][r]
        gone += first
    assert gone or window + new > 900
    got = []
    for table in (b.table, fewer):
        out, lse = torch.empty_like(q), torch.empty(3 * new, heads, device="cuda")
        ptq.cache_attention(out, q, cache, _c(table), _c(lens), _c(np.arange(4) * new), new, 0.125, ptq.Workspace(), st, causal=causal, window=window, lse=lse)
        ptq.check_status(st)
        got.append((out, lse))
    assert torch.equal(got[0][0], got[1][0]) and torch.equal(got[0][1], got[1][1])


@pytest.mark.parametrize("new,n", [(1, 90), (1, 3000), (40, 90), (90, 3000)])
@pytest.mark.parametrize("power", [8, 20, 23, 24, 26, 31, 60, 100, -24, -60])
def test_scores_of_any_size(power, new, n):
    """Whole numbers in q and k, a power of two for the scale: scores are exact, and from 2^8 on the keys with the largest one share the
    output.  The sum over them is exact but for fp16's and float32's rounding of what is added: (2^-11 + n 2^-23) of the mean of |v|,
    then the rounding of bf16."""
    heads, kv, dim, page = 4, 1, 64, 16
    scale = 2.0 ** power if power > 0 else -2.0 ** -power
    rng = np.random.default_rng(n + new)
    k = rng.integers(-8, 8, (n, kv, dim)).astype(np.float32)
    k[..., 0::32], k[..., 1::32] = -8, 7                          # steps of 1: whole numbers are held as they are
    v = rng.standard_normal((n, kv, dim)).astype(np.float32)
    q = rng.integers(-3, 4, (new, heads, dim))
    q[..., 0::32] = q[..., 1::32] = 0
    assert np.array_equal(ref.held4(k), k)
    cache, st = ptq.Cache4(-(-n // page), page, kv, dim), ptq.new_status()
    ptq.cache_append(cache, torch.from_numpy(k).cuda(), torch.from_numpy(v).cuda(), _c(np.arange(n)), st)
    out, lse = torch.empty(new, heads, dim, dtype=torch.bfloat16, device="cuda"), torch.empty(new, heads, device="cuda")
    ptq.cache_attention(out, torch.from_numpy(q).to(torch.bfloat16).cuda(), cache, _c([np.arange(-(-n // page))]), _c([n]), _c([0, new]), new, scale,
                        ptq.Workspace(), st, lse=lse)
    ptq.check_status(st)
    got, got_lse, held = out.cpu().double().numpy(), lse.cpu().double().numpy(), ref.held4(v)[:, 0]
    for i in range(0, new, 7):
        for h in range(heads):
            x = np.sign(scale) * (k[:n - new + i + 1, 0].astype(np.int64) @ q[i, h])
            best = held[:len(x)][x == x.max()]
            want, mass = best.mean(0), np.abs(best).mean(0)
            assert (np.abs(got[i, h] - want) <= (2.0 ** -11 + n * 2.0 ** -23 + 2.0 ** -20) * mass + 2.0 ** -8 * np.abs(want)).all()
            exact = float(x.max()) * abs(scale) + np.log(len(best))
            assert abs(got_lse[i, h] - exact) <= 2.0 ** -21 * (2 + abs(exact))


class _Attention:
    """Attention of the last tokens of a few requests, sized so that more rows need a larger workspace."""

    def __init__(self, seed):
        self.heads, self.dim, page, n = 8, 64, 16, 700
        g = base._gen(seed)
        self.n, self.cache, self.st = n, ptq.Cache4(-(-n // page), page, 2, self.dim), ptq.new_status()
        x = torch.randn(n, 2, self.dim, generator=g).cuda()
        ptq.cache_append(self.cache, x, x.flip(0), _c(np.arange(n)), self.st)
        self.table, self.lens = _c([np.arange(-(-n // page))]), _c([n])
        self.q = torch.randn(300, self.heads, self.dim, generator=g).to(torch.float16).cuda()

    def __call__(self, out, new, ws, stream=None):
        ptq.cache_attention(out, self.q[:new], self.cache, self.table, self.lens, self.cu[new], new, 0.125, ws, self.st, stream=stream)

    def outputs(self, *news):
        self.cu = {n: _c([0, n]) for n in news}
        return [torch.full((n, self.heads, self.dim), 7.0, dtype=torch.float16, device="cuda") for n in news]


def test_a_captured_call_keeps_its_scratch_when_others_need_more():
    job, ws = _Attention(1), ptq.Workspace()
    few, many, want = job.outputs(1, 300, 1)
    job(want, 1, ptq.Workspace())
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        job(few, 1, ws)
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        job(few, 1, ws)
    first, size = ws.buf.data_ptr(), ws.buf.numel()
    job(many, 300, ws)
    assert ws.buf.numel() > size and ws.buf.data_ptr() != first
    others = [torch.full((size,), 0x5A, dtype=torch.uint8, device="cuda") for _ in range(4)]       # the freed buffer's size
    assert all(o.data_ptr() != first for o in others)
    for _ in range(3):
        few.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(few, want) and all((o == 0x5A).all() for o in others)
    ptq.check_status(job.st)


def test_scratch_of_another_stream_is_not_given_away_while_it_is_used():
    job = _Attention(2)
    few, many, want, want_many = job.outputs(1, 300, 1, 300)
    job(want, 1, ptq.Workspace())
    job(want_many, 300, ptq.Workspace())
    ws, side = ptq.Workspace(), torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(50_000_000)                              # some 25 ms in which nothing of what follows runs there
    job(few, 1, ws, stream=side)
    size, first = ws.buf.numel(), ws.buf.data_ptr()
    job(many, 300, ws, stream=side)                                # a larger buffer: the first one is free for `side` alone
    others = [torch.full((size,), 0x5A, dtype=torch.uint8, device="cuda") for _ in range(4)]
    assert all(o.data_ptr() != first for o in others) and not side.query()
    used = ws.buf.data_ptr(), ws.buf.numel()
    del ws
    others += [torch.full((used[1],), 0x5A, dtype=torch.uint8, device="cuda") for _ in range(2)]
    assert all(o.data_ptr() != used[0] for o in others)
    torch.cuda.synchronize()
    ptq.check_status(job.st)
    assert torch.equal(few, want) and torch.equal(many, want_many) and all((o == 0x5A).all() for o in others)


def test_scratch_made_on_one_stream_and_used_on_another_is_not_given_away():
    job, ws = _Attention(3), ptq.Workspace()
    few, want = job.outputs(1, 1)
    job(want, 1, ws)                                               # made on the current stream
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(50_000_000)
    job(few, 1, ws, stream=side)
    size, first = ws.buf.numel(), ws.buf.data_ptr()
    del ws
    others = [torch.full((size,), 0x5A, dtype=torch.uint8, device="cuda") for _ in range(4)]
    assert all(o.data_ptr() != first for o in others) and not side.query()
    torch.cuda.synchronize()
    assert torch.equal(few, want) and all((o == 0x5A).all() for o in others)


def test_rows_of_one_shape_may_alternate_in_a_buffer():
    heads, kv, dim, page, n = 8, 2, 64, 16, 90
    g = base._gen(5)
    cache, st = ptq.Cache4(6, page, kv, dim), ptq.new_status()
    x = torch.randn(n, kv, dim, generator=g).cuda()
    ptq.cache_append(cache, x, x.flip(0), _c(np.arange(n)), st)
    both = torch.full((n, kv, 2, dim), 9.0, device="cuda")
    apart = [torch.empty(n, kv, dim, device="cuda") for _ in range(2)]
    ptq.cache_read(cache, _c(np.arange(n)), both[:, :, 0], both[:, :, 1], st)
    ptq.cache_read(cache, _c(np.arange(n)), *apart, st)
    assert torch.equal(both[:, :, 0], apart[0]) and torch.equal(both[:, :, 1], apart[1])
    args = cache, _c([np.arange(6)]), _c([n]), _c([0, 40]), 40, 0.125, ptq.Workspace(), st
    q = torch.randn(40, heads, dim, generator=g).to(torch.bfloat16).cuda()
    want = torch.empty_like(q)
    ptq.cache_attention(want, q, *args)
    for shape, part in (((40, 2, heads, dim), lambda t, i: t[:, i]), ((40, heads, 2, dim), lambda t, i: t[:, :, i]), ((heads, 40, 2, dim), lambda t, i: t[:, :, i].transpose(0, 1))):
        buf = torch.full(shape, 9.0, dtype=torch.bfloat16, device="cuda")
        part(buf, 0).copy_(q)
        ptq.cache_attention(part(buf, 1), part(buf, 0), *args)
        assert torch.equal(part(buf, 1), want) and torch.equal(part(buf, 0), q)
    ptq.check_status(st)


@pytest.mark.parametrize("k", [1, 100, 129, 5000])
def test_a_single_row_has_no_stride(k):
    """Contiguous operands of one row, of any length: the stride of a single row is never used."""
    x, w = torch.randn(1, k, generator=base._gen(k)).cuda(), torch.randn(1, k, generator=base._gen(k + 1)).cuda()
    st, got = ptq.new_status(), []
    for t, rows in ((x, 1), (w, 128)):
        q, s = torch.empty(1, k, dtype=torch.float8_e4m3fn, device="cuda"), torch.empty(1, -(-k // 128), device="cuda")
        ptq.fp8_quantize(t, q, s, st, block_rows=rows)
        rq, rs = ref.f8_cast(t.cpu().double().numpy(), rows)
        assert np.array_equal(q.cpu().double().numpy(), rq) and np.array_equal(s.cpu().double().numpy(), rs)
        got += [q, s]
    C = torch.empty(1, 1, device="cuda")
    ptq.fp8_matmul(C, *got, st)
    ptq.check_status(st)
    base._check_product(C, *got)


def test_calls_wait_for_copies_and_for_other_streams():
    """The kernels are put in place early; what a copy, another stream's work or an ordinary kernel before them wrote has to be there."""
    m, k = 4096, 2048
    st = ptq.new_status()
    x, q, s = torch.zeros(m, k, device="cuda"), ptq.fp8_empty(m, k), torch.empty(m, k // 128, device="cuda")
    hosts = [torch.randn(m, k, generator=base._gen(i)).pin_memory() for i in range(3)]
    want = []
    for h in hosts:
        ptq.fp8_quantize(h.cuda(), q, s, st)
        want.append((q.view(torch.uint8).clone(), s.clone()))
    side, got = torch.cuda.Stream(), []
    for i, h in enumerate(hosts * 2):
        qq, ss = ptq.fp8_empty(m, k), torch.empty(m, k // 128, device="cuda")
        ptq.fp8_quantize(x, q, s, st)                              # puts its successor in place early
        if i < 3:
            x.copy_(h, non_blocking=True)
        else:
            side.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(side):
                torch.cuda._sleep(2_000_000)
                x.copy_(h, non_blocking=True)
            torch.cuda.current_stream().wait_stream(side)
        ptq.fp8_quantize(x, qq, ss, st)
        got.append((qq, ss))
    torch.cuda.synchronize()
    ptq.check_status(st)
    for i, (qq, ss) in enumerate(got):
        assert torch.equal(qq.view(torch.uint8), want[i % 3][0]) and torch.equal(ss, want[i % 3][1]), i


def test_a_capture_that_forks_and_joins():
    """Casts, products and attention on two streams of one captured graph, replayed with other inputs."""
    heads, kv, dim, page, n = 8, 2, 64, 16, 500
    st, g = ptq.new_status(), base._gen(8)
    cache = ptq.Cache4(40, page, kv, dim)
    cache.pages.zero_()
    x = torch.randn(n, kv, dim, generator=g).cuda()
    ptq.cache_append(cache, x, x.flip(0), _c(np.arange(n)), st)
    B, sb = base._cast(torch.randn(heads * dim, 700, generator=g).cuda(), 128, st)
    a = torch.zeros(96, 700, dtype=torch.bfloat16, device="cuda")
    A, sa = ptq.fp8_empty(96, 700), torch.empty(96, 6, device="cuda")
    q, out = torch.empty(96, heads, dim, dtype=torch.bfloat16, device="cuda"), torch.empty(96, heads, dim, dtype=torch.bfloat16, device="cuda")
    new = torch.zeros(96, kv, dim, dtype=torch.bfloat16, device="cuda")
    lens, slots, table, cu, ws = _c([n + 96]), _c(np.arange(n, n + 96)), _c([np.arange(40)]), _c([0, 96]), ptq.Workspace()
    side, main = torch.cuda.Stream(), torch.cuda.Stream()

    def step(s):
        side.wait_stream(s)
        ptq.fp8_quantize(a, A, sa, st, stream=s)
        ptq.cache_append(cache, new, new, slots, st, stream=side)
        ptq.fp8_matmul(q.flatten(1), A, sa, B, sb, st, stream=s)
        s.wait_stream(side)
        ptq.cache_attention(out, q, cache, table, lens, cu, 96, 0.125, ws, st, stream=s)

    main.wait_stream(torch.cuda.current_stream())
    step(main)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=main):
        step(main)
    for i in range(4):
        a.copy_(torch.randn(96, 700, generator=g))
        new.copy_(torch.randn(96, kv, dim, generator=g))
        out.fill_(7.0)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        got = out.clone()
        out.fill_(7.0)
        step(torch.cuda.current_stream())
        torch.cuda.synchronize()
        assert torch.equal(got, out) and torch.isfinite(got.float()).all()
    ptq.check_status(st)


@pytest.mark.parametrize("eager_first", [True, False])
def test_scratch_of_a_capture_may_be_made_before_it_or_in_it(eager_first):
    job, ws = _Attention(4), ptq.Workspace()
    few, many, want, want_many = job.outputs(1, 300, 1, 300)
    job(want, 1, ptq.Workspace())
    job(want_many, 300, ptq.Workspace())
    if eager_first:
        job(few, 1, ws)                                            # on the current stream; the capture is on another one
    torch.cuda.synchronize()
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(graph, stream=side):
        job(few, 1, ws)
    held = ws.buf.data_ptr()
    job(many, 300, ws)                                             # grows, eagerly
    assert ws.buf.data_ptr() != held
    others = [torch.full((1 << 24,), 0x5A, dtype=torch.uint8, device="cuda") for _ in range(4)]
    for _ in range(3):
        few.fill_(7.0)
        many.fill_(7.0)
        graph.replay()
        job(many, 300, ws)
        torch.cuda.synchronize()
        assert torch.equal(few, want) and torch.equal(many, want_many) and all((o == 0x5A).all() for o in others)
    ptq.check_status(job.st)
    del graph, ws
    torch.cuda.synchronize()
