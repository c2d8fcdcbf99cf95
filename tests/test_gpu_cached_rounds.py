"""Weights of a paged cache's slots where a workgroup takes several rounds of them: its place in LDS is used again for the next ones."""
import pathlib
import re

import pytest
import torch

import cached_ref as ref
from test_gpu_cached import gpu, near
from test_gpu_cached_long import weigh_64

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
CSRC = pathlib.Path(__file__).resolve().parent.parent / "paper_2603_09215_amd" / "csrc"


def rounds(n, nkv, length, table_slots, dtype):
    """that the longest of n sequences takes a workgroup of the kernel for many rows (csrc/cached_ops.hip)"""
    cap = re.search(r"Weigh<T, true>::WAVES, std::max\(1, \(1 << (\d+)\) / heads\), lds\)", (CSRC / "cached_ops.hip").read_text())
    assert cap, "the launch has changed: so has this test to"
    each, heads = 2 if dtype is BF16 else 1, n * nkv
    grid = min(-(-(-(-table_slots // 32)) // each), max(1, (1 << int(cap[1])) // heads))
    return -(-(-(-length // 32)) // (each * grid))


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("hd", [64, 128])
def test_several_rounds(hd, dtype):
    """1024 sequences of 8 heads, some of them of up to 2000 slots: the same bits as in a batch of three, whose grid has a workgroup for each piece, and near the formula's"""
    c, n, nkv, rows, group, page = gpu(), 1024, 8, 64, 4, 64
    g = torch.Generator(device="cuda").manual_seed(71)
    i32 = dict(dtype=torch.int32, device="cuda")
    pool = torch.randn(64, 1, 2, nkv, page, hd, generator=g, device="cuda").to(dtype)
    q = torch.randn(n * rows, nkv * group, hd, generator=g, device="cuda").to(dtype)
    table = torch.randint(0, 64, (n, 32), generator=g, **i32)
    lengths = torch.randint(rows, 200, (n,), generator=g, **i32)
    long = {0: 2000, 2: 1503, 500: 1999, 501: 1025, n - 1: 1797}
    for s, length in long.items():
        lengths[s] = length
        assert rounds(n, nkv, length, 2048, dtype) >= 3 and rounds(3, nkv, length, 2048, dtype) == 1
    cache, batch = c.PagedCache(pool), c.CachedRows(torch.arange(n + 1, **i32) * rows, lengths, table)
    lse = torch.empty(n * rows, nkv * group, device="cuda")
    c.cached_attend(q, cache, batch, lse=lse)
    weights = c.cached_weigh(q, lse, cache, batch)
    assert torch.equal(weights, c.cached_weigh(q, lse, cache, batch))
    for s in (0, 500, n - 3):
        some = c.CachedRows(torch.arange(4, **i32) * rows, lengths[s:s + 3].contiguous(), table[s:s + 3].contiguous())
        part = slice(s * rows, (s + 3) * rows)
        assert torch.equal(weights[s:s + 3], c.cached_weigh(q[part], lse[part], cache, some))
        b = ref.Batch([0, rows, 2 * rows, 3 * rows], lengths[s:s + 3].tolist(), table[s:s + 3].tolist(), 3 * rows, 64, page)
        want, tol = weigh_64(q[part], lse[part], pool, b, hd ** -0.5, True)
        near(weights[s:s + 3], want, tol, f"sequences from {s}")


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_several_rounds_of_single_steps(dtype):
    """the kernel for few rows, whose waves go through their slots by themselves"""
    c, n, nkv, nq, hd, page = gpu(), 300, 4, 8, 64, 64
    g = torch.Generator(device="cuda").manual_seed(72)
    i32 = dict(dtype=torch.int32, device="cuda")
    pool = torch.randn(64, 1, 2, nkv, page, hd, generator=g, device="cuda").to(dtype)
    q = torch.randn(n, nq, hd, generator=g, device="cuda").to(dtype)
    table, lengths = torch.randint(0, 64, (n, 40), generator=g, **i32), torch.randint(1, 2561, (n,), generator=g, **i32)
    cache, batch = c.PagedCache(pool), c.CachedRows(torch.arange(n + 1, **i32), lengths, table)
    lse = torch.empty(n, nq, device="cuda")
    c.cached_attend(q, cache, batch, lse=lse)
    weights = c.cached_weigh(q, lse, cache, batch)
    for s in (0, 150, n - 2):
        b = ref.Batch([0, 1, 2], lengths[s:s + 2].tolist(), table[s:s + 2].tolist(), 2, 64, page)
        want, tol = weigh_64(q[s:s + 2], lse[s:s + 2], pool, b, hd ** -0.5, True)
        near(weights[s:s + 2], want, tol, f"sequences from {s}")
