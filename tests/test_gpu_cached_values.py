"""Attention over a paged cache: values that are no numbers, in slots that every row sees, under probabilities that fp32 has as zero."""
import math

import pytest
import torch

import cached_ref as ref
from test_gpu_cached import gpu, make_batch, near, rows_of
from test_gpu_cached_long import attend_64, full_pool

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16

# (rows, length), query heads, kv heads, head_dim, type: streams and both tiles, in one part and in several
KINDS = [([(1, 120)], 28, 4, 128, BF16), ([(1, 3000)], 7, 1, 128, BF16), ([(5, 90), (1, 100)], 4, 2, 64, BF16), ([(900, 901)], 14, 2, 64, BF16),
         ([(300, 1000)], 28, 4, 128, BF16), ([(2500, 2600)], 28, 4, 128, BF16), ([(1, 2000)], 7, 1, 128, F32), ([(30, 60)], 4, 2, 64, F32)]


@pytest.mark.parametrize("value", [math.inf, -math.inf, math.nan])
@pytest.mark.parametrize("shape,nq,nkv,hd,dtype", KINDS)
def test_no_numbers_under_probabilities_of_zero(shape, nq, nkv, hd, dtype, value):
    """slot 3, e^-140 of the others: its infinity or NaN is its element's result in all rows that see it, and every other element is as if it were none"""
    c, page, slot, element = gpu(), 16, 3, hd - 3
    starts, lengths, table, pages, m = make_batch(shape, page, 81)
    b = ref.Batch(starts, lengths, table, m, pages, page)
    pool, q = full_pool(pages, 1, nkv, page, hd, dtype, 82), rows_of(m, nq, hd, dtype, 83)
    q[:, :, 0] = 4.0
    for s in range(b.n):
        at = b.page(s, slot)
        pool[at, 0, 0, :, slot] = 0.0
        pool[at, 0, 0, :, slot, 0] = -35.0 * hd ** 0.5
        pool[at, 0, 1, :, slot, element] = 0.0
    want, tol, want_lse, lse_tol = attend_64(q, pool, b, 0, hd ** -0.5, True)
    for s in range(b.n):
        pool[b.page(s, slot), 0, 1, :, slot, element] = value
    lse = torch.empty(m, nq, device="cuda")
    got = c.cached_attend(q, c.PagedCache(pool), c.CachedRows(starts.cuda(), lengths.cuda(), table.cuda()), lse=lse)
    near(lse, want_lse, lse_tol, "lse")
    for s in range(b.n):
        first = b.row0[s] + max(0, slot - b.slot(s, 0))   # the row that sees it first
        hit = got[first:b.row0[s] + b.rows[s], :, element].float()
        assert bool(hit.isnan().all()) if math.isnan(value) else bool((hit == value).all())
        want[first:b.row0[s] + b.rows[s], :, element] = math.nan   # (not compared)
    near(got, want, tol, "out")
