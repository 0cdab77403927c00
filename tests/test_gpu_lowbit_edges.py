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
