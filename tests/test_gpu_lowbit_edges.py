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
