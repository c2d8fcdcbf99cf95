"""Attention over a paged cache whose values are near the end of their type's range: sums before the division would leave it."""
import pytest
import torch

import cached_ref as ref
from test_gpu_cached import gpu, make_batch, near, rows_of
from test_gpu_cached_long import attend_64, full_pool
from test_gpu_cached_values import KINDS

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16


@pytest.mark.parametrize("shape,nq,nkv,hd,dtype", KINDS + [([(1, 30000)], 8, 1, 128, BF16), ([(500, 2000)], 28, 4, 128, BF16)])
def test_values_up_to_2_127(shape, nq, nkv, hd, dtype):
    c, page = gpu(), 64
    starts, lengths, table, pages, m = make_batch(shape, page, 85)
    b = ref.Batch(starts, lengths, table, m, pages, page)
    pool, q = full_pool(pages, 1, nkv, page, hd, dtype, 86), rows_of(m, nq, hd, dtype, 87)
    values = pool[:, :, 1].float()
    pool[:, :, 1] = (values / values.abs().max() * 2.0 ** 127).to(dtype)
    pool[:, :, 1, :, :, ::2] = pool[:, :, 1, :, :, ::2].abs()   # (every second element of one sign: its sums do not cancel)
    lse = torch.empty(m, nq, device="cuda")
    got = c.cached_attend(q, c.PagedCache(pool), c.CachedRows(starts.cuda(), lengths.cuda(), table.cuda()), lse=lse)
    want, tol, want_lse, lse_tol = attend_64(q, pool, b, 0, hd ** -0.5, True)
    near(lse, want_lse, lse_tol, "lse")
    near(got, want, tol, "out")


@pytest.mark.parametrize("shape,nq,nkv,hd,dtype", [([(1, 3000)], 7, 1, 128, BF16), ([(500, 2000)], 28, 4, 128, BF16), ([(1200, 1300)], 28, 4, 64, BF16), ([(2500, 2600)], 28, 4, 128, BF16),
                                                  ([(1, 2000)], 7, 1, 128, F32)])
def test_large_values_of_some_slots_and_one_element(shape, nq, nkv, hd, dtype):
    """in the first 100 slots, so in some of the parts alone: that element's results are the formula's, and the others' the bits that they are without"""
    c, page = gpu(), 64
    starts, lengths, table, pages, m = make_batch(shape, page, 88)
    b = ref.Batch(starts, lengths, table, m, pages, page)
    pool, q = full_pool(pages, 1, nkv, page, hd, dtype, 89), rows_of(m, nq, hd, dtype, 90)
    batch = c.CachedRows(starts.cuda(), lengths.cuda(), table.cuda())
    lse, clean_lse = torch.empty(m, nq, device="cuda"), torch.empty(m, nq, device="cuda")
    clean = c.cached_attend(q, c.PagedCache(pool), batch, lse=clean_lse)
    for t in range(100):
        pool[b.page(0, t), 0, 1, :, t % page, 7] = 2.0 ** 127
    got = c.cached_attend(q, c.PagedCache(pool), batch, lse=lse)
    rest = torch.arange(hd, device="cuda") != 7
    assert torch.equal(got[:, :, rest], clean[:, :, rest]) and torch.equal(lse, clean_lse)
    want, tol, _, _ = attend_64(q, pool, b, 0, hd ** -0.5, True)
    near(got, want, tol, "out")
