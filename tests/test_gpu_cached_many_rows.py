"""Weights of a paged cache's slots from many rows: what their sums are off by does not grow with their number."""
import math

import pytest
import torch

import cached_ref as ref
from test_gpu_cached import gpu

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("nq,nkv,hd,n", [(16, 1, 128, 1), (16, 2, 64, 1), (1, 1, 64, 1), (1, 1, 128, 200)])
def test_sums_of_many_rows(nq, nkv, hd, n, dtype):
    """queries of zeros: every row gives each slot exp(-lse), the same number, whose additions one by one round the same way for long.  (Many pairs of a sequence, whose
    blocks the waves share, and 200 sequences of fewer, where each wave has its own slots.)"""
    c = gpu()
    rows, page = 8192 if n == 1 else 250, 64
    i32 = dict(dtype=torch.int32, device="cuda")
    pages = rows // page + 1
    pool = torch.zeros(pages, 1, 2, nkv, page, hd, dtype=dtype, device="cuda")
    batch = c.CachedRows(torch.arange(n + 1, **i32) * rows, torch.full((n,), rows, **i32), torch.arange(pages, **i32).expand(n, -1).contiguous())
    q = torch.zeros(n * rows, nq, hd, dtype=dtype, device="cuda")
    u, worst = ref.U, 0.0
    for value in (0.3, 1.0 / 3, 1.1, 0.7):
        lse = torch.full((n * rows, nq), value, device="cuda")
        got = c.cached_weigh(q, lse, c.PagedCache(pool), batch, causal=False)[:, :, :rows].double()
        want = rows * (nq // nkv) * math.exp(-float(torch.tensor(value)))
        # a probability: 2 |lse| log2 e rounded, the exponential's steps; sixteen added in a lane, sums of blocks with what their additions lose, two halves
        # and eight waves
        tol = want * ((4 + 3 * value) * 2 + 16 + 4 + 1 + 8) * u
        worst = max(worst, float((got - want).abs().max()) / tol)
    assert worst <= 1, worst


def test_infinite_sums_stay_infinite():
    """an lse far below a row's sum, which no pass of attention leaves: weights past fp32's range are infinite, the others as they are"""
    c, rows = gpu(), 600
    i32 = dict(dtype=torch.int32, device="cuda")
    pool = torch.zeros(10, 1, 2, 1, 64, 64, device="cuda")
    batch = c.CachedRows(torch.tensor([0, rows], **i32), torch.tensor([rows], **i32), torch.arange(10, **i32).view(1, 10))
    lse = torch.zeros(rows, 4, device="cuda")
    lse[100] = -200.0
    got = c.cached_weigh(torch.zeros(rows, 4, 64, device="cuda"), lse, c.PagedCache(pool), batch)[0, 0, :rows]
    assert bool((got[:101] == math.inf).all())
    want = 4.0 * torch.arange(rows - 101, 0, -1, device="cuda")
    assert bool(((got[101:] - want).abs() <= 64 * ref.U * want).all())
