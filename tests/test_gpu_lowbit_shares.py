"""The low-bit serving operators where a worker has much to do: many k blocks a CTA, many chunks of keys a warp or CTA, several
pieces of row tiles one after another, a running maximum that rises far from chunk to chunk, and calls that run at the same time.
Against the definitions in 64 bits, with the tolerances of ``test_gpu_lowbit``."""
import numpy as np
import pytest
import torch

import lowbit_ref as ref
import test_gpu_lowbit as base
from paper_2509_05576_b200 import ptq

pytestmark = pytest.mark.gpu


def _c(v):
    return torch.tensor(np.asarray(v, np.int32), device="cuda")


def _sms():
    return min(160, torch.cuda.get_device_properties(0).multi_processor_count)


# --------------------------------------------------------------------------------------------------------- many k blocks
# rows that go to the persistent kernel (scales in rows of whole 16-byte pieces and not, a last group of four that is partial) and
# to the kernel for few rows with more than sixteen blocks for a CTA
@pytest.mark.parametrize("m,n,k", [(2100, 2500, 1024), (1500, 1300, 1300), (700, 5000, 4096), (2049, 1027, 1664), (1, 11008, 4096), (40, 11008, 4200),
                                   (70, 9000, 4500), (17, 20000, 2500)])
def test_product_of_many_k_blocks(m, n, k):
    A, sa, B, sb = base._operands(m, n, k, m + k, power=False)
    C = torch.full((m, n), float("nan"), device="cuda")
    st = ptq.new_status()
    ptq.fp8_matmul(C, A, sa, B, sb, st)
    ptq.check_status(st)
    base._check_product(C, A, sa, B, sb)


# --------------------------------------------------------------------------------------------------------- many chunks
class Stairs:
    """Keys whose scores climb by more than 2^7 twice and fall again, with values that make up for it: every part of the sequence
    weighs about the same in the output.  All requests read the same pages, each as far as its length."""

    def __init__(self, n, kv_heads, dim, page, seed):
        rng = np.random.default_rng(seed)
        level = np.select([np.arange(n) < 400, np.arange(n) < 800, np.arange(n) < 1100], [0.0, 7.6, 15.0], 0.3)       # log2
        self.way = rng.choice([-1.0, 1.0], (kv_heads, dim))
        a = level * np.log(2) / dim ** 0.5
        k = a[:, None, None] * self.way + 0.05 * rng.standard_normal((n, kv_heads, dim))
        v = np.exp2(14.5 - level)[:, None, None] * rng.uniform(0.2, 1.0, (n, kv_heads, dim))
        pages = -(-n // page)
        self.cache = ptq.Cache4(pages + 1, page, kv_heads, dim)
        self.order = rng.permutation(pages + 1)[:pages]
        j = np.arange(n)
        st = ptq.new_status()
        k, v = k.astype(np.float32), v.astype(np.float32)
        ptq.cache_append(self.cache, torch.from_numpy(k).cuda(), torch.from_numpy(v).cuda(), _c(self.order[j // page] * page + j % page), st)
        ptq.check_status(st)
        self.keys, self.values, self.rng = ref.held4(k), ref.held4(v), rng

    def check(self, lens, new, ratio, dtype, rows_of):
        """Attention of every request's last `new` rows; the rows that rows_of(request) names against the definition."""
        kv, dim = self.way.shape
        heads, total = kv * ratio, len(lens) * new
        q = np.repeat(self.way, ratio, 0) * (1 + 0.02 * self.rng.standard_normal((total, heads, 1))) + 0.3 * self.rng.standard_normal((total, heads, dim))
        q = torch.from_numpy(q).to(dtype)
        out, lse, st = torch.empty(total, heads, dim, dtype=dtype, device="cuda"), torch.empty(total, heads, device="cuda"), ptq.new_status()
        table = _c(np.tile(self.order, (len(lens), 1)))
        ptq.cache_attention(out, q.cuda(), self.cache, table, _c(lens), _c(np.arange(len(lens) + 1) * new), new, dim ** -0.5, ptq.Workspace(), st, lse=lse)
        ptq.check_status(st)
        got, got_lse, top = out.cpu().double().numpy(), lse.cpu().double().numpy(), np.abs(self.values).max()
        for r, n in enumerate(lens):
            for i in rows_of(r):
                sees, at = n - new + i + 1, r * new + i
                want, want_lse, mass, reach = ref.attention(q[at:at + 1].double().numpy(), self.keys[:sees], self.values[:sees], sees, dim ** -0.5, True, 0)
                d = (dim + 4) * 2.0 ** -23 * reach
                tol = ((2 * d + 2.0 ** -21)[..., None] + 2.0 ** -11 + sees * 2.0 ** -23) * mass + base.HALF_STEP[dtype] * np.abs(want) + sees * 2.0 ** -33 * top
                off = np.abs(got[at] - want[0])
                assert (off <= tol[0]).all(), (r, i, float((off - tol[0]).max()))
                assert (np.abs(got_lse[at] - want_lse[0]) <= d[0] + sees * 2.0 ** -23 + 2.0 ** -21 * (2 + np.abs(want_lse[0]))).all()


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("ratio", [4, 12, 16])
def test_single_tokens_with_many_chunks_a_warp(ratio, dim, dtype):
    s = Stairs(2000, 8, dim, 64, ratio + dim)
    lens = [1300 + 37 * i % 700 for i in range(56)] + [5, 0, 64, 65, 2000]
    warps = 12 if ratio <= 8 else 8
    units = 8 * sum(max(-(-n // 64), 1) + 1 for n in lens) * (1 if ratio <= 16 else 2)
    assert units >= 5 * warps * _sms()                            # chunks a warp: pieces of several chunks, several pieces
    s.check(lens, 1, ratio, dtype, lambda r: [0] if lens[r] and r % 7 in (0, 3) else [])


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
@pytest.mark.parametrize("dim,ratio,new", [(128, 4, 300), (64, 8, 300), (128, 7, 90), (64, 3, 700)])
def test_prompts_with_many_chunks_a_cta(dim, ratio, new, dtype):
    s = Stairs(3400, 8, dim, 64, ratio + dim)
    lens = [3400, 2900, 1500]
    units = 8 * sum(-(-new * ratio // 256) * ((n - new) // 128 + 1) for n in lens)
    assert units >= 5 * _sms()
    picks = [0, 1, new // 2, new - 1] + [int(x) for x in np.random.default_rng(3).integers(0, new, 4)]
    s.check(lens, new, ratio, dtype, lambda r: picks)


def test_few_rows_keep_small_probabilities():
    """One key on top and thousands 2^-36 below it with large values: the kernel for few rows holds probabilities times 2^15, so
    that what rounding to fp16 takes is at most half a step of 2^-24, 2^-40 of the largest, a key."""
    n, dim = 6000, 64
    k, v = np.zeros((n, 1, dim), np.float32), np.full((n, 1, dim), 31680.0, np.float32)
    k[777], v[777] = 36 * np.log(2) / 8, 0.0
    cache = ptq.Cache4(6, 1024, 1, dim)
    st = ptq.new_status()
    ptq.cache_append(cache, torch.from_numpy(k).cuda(), torch.from_numpy(v).cuda(), _c(np.arange(n)), st)
    q = torch.ones(1, 1, dim, dtype=torch.float16)
    out = torch.empty(1, 1, dim, dtype=torch.float16, device="cuda")
    ptq.cache_attention(out, q.cuda(), cache, _c([np.arange(6)]), _c([n]), _c([0, 1]), 1, 0.125, ptq.Workspace(), st)
    ptq.check_status(st)
    want, _, mass, reach = ref.attention(q.double().numpy(), ref.held4(k), ref.held4(v), n, 0.125, True, 0)
    tol = (2 * (dim + 4) * 2.0 ** -23 * reach[..., None] + 2.0 ** -11 + n * 2.0 ** -23) * mass + 2.0 ** -11 * want + n * 2.0 ** -40 * 31680
    assert (np.abs(out.cpu().double().numpy() - want) <= tol).all() and want.min() > 50 * n * 2.0 ** -40


# ---------------------------------------------------------------------------------------------------------- side by side
def test_calls_that_run_at_the_same_time_do_not_meet():
    """Attention of single tokens, of prompts, and products, queued on three streams without a wait between them."""
    heads, kv, dim, page = 16, 4, 64, 32
    rng = np.random.default_rng(9)
    lens, jobs = [2500, 900, 40], []
    for new in ([1, 1, 1], [300, 20, 3]):
        cache = ptq.Cache4(200, page, kv, dim)
        st = ptq.new_status()
        x = torch.from_numpy(rng.standard_normal((200 * page, kv, dim)).astype(np.float32)).cuda()
        ptq.cache_append(cache, x, x.flip(0), _c(np.arange(200 * page)), st)
        table = _c(rng.permutation(200)[:180].reshape(3, 60).repeat(2, 1)[:, :90])
        q = torch.from_numpy(rng.standard_normal((sum(new), heads, dim))).to(torch.bfloat16).cuda()
        args = (q, cache, table, _c(lens), _c(np.concatenate([[0], np.cumsum(new)])), max(new), 0.125, ptq.Workspace(), st)
        jobs.append((lambda out, lse, s, a=args: ptq.cache_attention(out, *a, lse=lse, stream=s), q, st))
    operands = [base._operands(m, 1100, 700, m) for m in (16, 2100)]
    st3 = ptq.new_status()

    def products(outs, s):
        for C, o in zip(outs, operands):
            ptq.fp8_matmul(C, *o, st3, stream=s)

    def attention(i, s=None):
        out, lse = torch.empty_like(jobs[i][1]), torch.empty(jobs[i][1].shape[:2], device="cuda")
        return out, lse

    outs = lambda: [torch.empty(o[0].shape[0], 1100, device="cuda") for o in operands]  # noqa: E731
    want = [attention(0), attention(1)]
    want_c = outs()
    for i in range(2):
        jobs[i][0](*want[i], None)
    products(want_c, None)
    rounds = 12
    got = [[attention(0), attention(1), outs()] for _ in range(rounds)]
    streams = [torch.cuda.Stream() for _ in range(3)]
    torch.cuda.synchronize()
    for g in got:
        jobs[0][0](*g[0], streams[0])
        jobs[1][0](*g[1], streams[1])
        products(g[2], streams[2])
    torch.cuda.synchronize()
    for st in (jobs[0][2], jobs[1][2], st3):
        ptq.check_status(st)
    for g in got:
        for i in range(2):
            assert torch.equal(g[i][0], want[i][0]) and torch.equal(g[i][1], want[i][1])
        assert torch.equal(g[2][0], want_c[0]) and torch.equal(g[2][1], want_c[1])
