"""Norms of queries and keys on their way into a paged cache, with gains and eps far from one."""
import pytest
import torch

import cached_ref as ref
from test_gpu_cached import gpu, make_batch, near, rows_of

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16


def normed(size, gain_size, eps, dtype, hd=64, rotary=0):
    c = gpu()
    starts, lengths, table, pages, m = make_batch([(5, 5)], 16, 2)
    b = ref.Batch(starts, lengths, table, m, pages, 16)
    q, k, v = (rows_of(m, h, hd, F32, 3 + i) * size for i, h in enumerate((3, 1, 1)))
    gain = (1 + torch.arange(hd) / hd) * gain_size
    pool = torch.zeros(pages, 1, 2, 1, 16, hd, dtype=dtype)
    want, tol, new, new_tol = ref.append(q.cpu(), k.cpu(), v.cpu(), pool, b, 0, rotary, False, ref.frequencies(rotary), 1.0, gain, gain, eps)
    cache = c.PagedCache(pool.cuda())
    got = c.cached_append(q, k, v, cache, c.CachedRows(starts.cuda(), lengths.cuda(), table.cuda()), rotation=c.Rotation(rotary), q_gain=gain.cuda(), k_gain=gain.cuda(), eps=eps)
    near(got, want, tol, "q")
    near(cache.pool, new, new_tol, "pool")


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("size,gain", [(1e-10, 1e30), (1e-12, 1e37), (1e15, 1e-30), (1e16, 1e-33), (1.0, 1e-33), (1.0, 1e37)])
def test_gains_far_from_one(size, gain, dtype):
    """a row's factor times its gain may leave fp32's range where the result is far from it"""
    normed(size, gain, 0.0, dtype)
    normed(size, gain, 0.0, dtype, hd=128, rotary=24)
