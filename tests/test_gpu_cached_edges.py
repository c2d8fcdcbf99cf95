"""The operators on a paged cache at the ends of their sizes: more slots than one round of workgroups weighs, as many heads as a call takes, and
a process whose first calls are captured."""
import os
import subprocess
import sys

import pytest
import torch

import cached_ref as ref
from test_gpu_cached import gpu, make_batch, near, rows_of
from test_gpu_cached_long import full_pool, weigh_64

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_weigh_more_slots_than_a_round(dtype):
    c = gpu()
    starts, lengths, table, pages, m = make_batch([(64, 270001)], 64, 61)
    b = ref.Batch(starts, lengths, table, m, pages, 64)
    pool = full_pool(pages, 1, 1, 64, 64, dtype, 62)
    q = rows_of(m, 4, 64, dtype, 63)
    lse = torch.empty(m, 4, device="cuda")
    cache, batch = c.PagedCache(pool), c.CachedRows(starts.cuda(), lengths.cuda(), table.cuda())
    c.cached_attend(q, cache, batch, lse=lse)
    weights = c.cached_weigh(q, lse, cache, batch)
    want, tol = weigh_64(q, lse, pool, b, 64 ** -0.5, True)
    near(weights, want, tol, "weights")


def test_evict_with_the_most_heads():
    """2^20 heads of sequences; pages for two of the sequences alone"""
    c = gpu()
    n, nkv, keep = 1 << 16, 16, 5
    g = torch.Generator(device="cuda").manual_seed(64)
    pool = torch.randn(8, 1, 2, nkv, 16, 128, generator=g, device="cuda")
    before = pool.clone()
    table = torch.full((n, 1), -1, dtype=torch.int32, device="cuda")
    table[12345], table[n - 1] = 6, 3
    lengths = torch.full((n,), 16, dtype=torch.int32, device="cuda")
    weights = torch.rand(n, nkv, 16, generator=g, device="cuda")
    out = torch.empty_like(weights)
    batch = c.CachedRows(torch.zeros(n + 1, dtype=torch.int32, device="cuda"), lengths, table)
    kept, left = c.cached_evict(c.PagedCache(pool), batch, weights, keep, first=1, recent=1, weights_out=out)
    order = 1 + weights[:, :, 1:15].argsort(dim=2, descending=True, stable=True)[:, :, :keep - 2]
    ends = torch.zeros(n, nkv, 2, dtype=torch.int64, device="cuda")
    ends[:, :, 1] = 15
    want = torch.cat([ends, order], dim=2).sort(dim=2).values
    assert torch.equal(kept.long(), want) and bool((left == keep).all())
    assert torch.equal(out[:, :, :keep], weights.gather(2, want)) and not bool(out[:, :, keep:].any())
    for s, page in ((12345, 6), (n - 1, 3)):
        for h in range(nkv):
            before[page, 0, :, h, :keep] = before[page, 0, :, h, want[s, h]]
    assert torch.equal(pool, before)


def test_long_tables_of_many_heads():
    """more heads times pieces of their tables than a launch has threads for: the same bits as in a batch of some of the sequences"""
    c = gpu()
    n, nkv, rows, group, hd, page = 1024, 8, 64, 4, 64, 64
    g = torch.Generator(device="cuda").manual_seed(66)
    i32 = dict(dtype=torch.int32, device="cuda")
    pool = torch.randn(64, 1, 2, nkv, page, hd, generator=g, device="cuda").to(BF16)
    q = torch.randn(n * rows, nkv * group, hd, generator=g, device="cuda").to(BF16)
    table = torch.randint(0, 64, (n, 1024), generator=g, **i32)
    lengths = torch.randint(rows, 200, (n,), generator=g, **i32)
    cache = c.PagedCache(pool)
    lse = torch.empty(n * rows, nkv * group, device="cuda")
    batch = c.CachedRows(torch.arange(n + 1, **i32) * rows, lengths, table)
    c.cached_attend(q, cache, batch, lse=lse)
    weights = c.cached_weigh(q, lse, cache, batch)
    for s in (0, 500, n - 3):
        some = c.CachedRows(torch.arange(4, **i32) * rows, lengths[s:s + 3].contiguous(), table[s:s + 3, :4].contiguous())
        part = slice(s * rows, (s + 3) * rows)
        want = c.cached_weigh(q[part], lse[part], cache, some)
        assert torch.equal(weights[s:s + 3, :, :256], want) and not bool(weights[s:s + 3, :, 256:].any())


def test_evict_to_other_pages_with_many_heads():
    c = gpu()
    n, nkv, page, pages, keep = 4096, 8, 64, 257, 16384
    g = torch.Generator(device="cuda").manual_seed(67)
    i32 = dict(dtype=torch.int32, device="cuda")
    pool = torch.randn(2 * pages, 1, 2, nkv, page, 128, generator=g, device="cuda").to(BF16)
    start = pool[:pages].clone()
    table, to = torch.full((n, pages), -1, **i32), torch.full((n, pages - 1), -1, **i32)
    lengths = torch.full((n,), 5, **i32)
    s = n - 2
    table[s], to[s], lengths[s] = torch.arange(pages, **i32), torch.arange(pages, 2 * pages - 1, **i32), pages * page
    weights = torch.zeros(n, nkv, pages * page, device="cuda")
    weights[s] = torch.rand(nkv, pages * page, generator=g, device="cuda")
    batch = c.CachedRows(torch.zeros(n + 1, **i32), lengths, table)
    kept, left = c.cached_evict(c.PagedCache(pool), batch, weights.clone(), keep, table_out=to)
    want = weights[s].argsort(dim=1, descending=True, stable=True)[:, :keep].sort(dim=1).values
    assert torch.equal(kept[s].long(), want) and int(left[s]) == keep and int(left[0]) == 5
    flat, moved = start[:, 0].permute(1, 2, 0, 3, 4).reshape(2, nkv, pages * page, 128), pool[pages:2 * pages - 1, 0].permute(1, 2, 0, 3, 4).reshape(2, nkv, keep, 128)
    for h in range(nkv):
        assert torch.equal(moved[:, h], flat[:, h, want[h]]), h
    assert torch.equal(pool[:pages], start)


@pytest.mark.parametrize("in_place", [True, False])
@pytest.mark.parametrize("kind", ["plain", "ties", "zeros", "nan"])
def test_evict_more_slots_than_a_workgroup_holds(kind, in_place):
    c = gpu()
    nkv, page, pages, keep, first, recent = 2, 32, 626, 9001, 5, 77
    length = page * pages - 3
    g = torch.Generator(device="cuda").manual_seed(68)
    i32 = dict(dtype=torch.int32, device="cuda")
    pool = torch.randn(pages + 300, 1, 2, nkv, page, 64, generator=g, device="cuda").to(BF16)
    start = pool.clone()
    weights = torch.randn(1, nkv, page * pages, generator=g, device="cuda")
    if kind == "ties":
        weights = torch.randint(0, 3, weights.shape, generator=g, device="cuda").float()
    elif kind == "zeros":
        weights = torch.where(weights < 0, 0.0, -0.0)
    elif kind == "nan":
        weights[weights > 1.5] = float("nan")
    given = weights.clone()
    order = torch.where(given.isnan(), float("inf"), given)[0, :, first:length - recent].argsort(dim=1, descending=True, stable=True)[:, :keep - first - recent] + first
    ends = torch.cat([torch.arange(first, device="cuda"), torch.arange(length - recent, length, device="cuda")])
    want = torch.cat([ends.expand(nkv, -1), order], dim=1).sort(dim=1).values
    table = torch.randperm(pages, generator=g, device="cuda").int().view(1, pages)
    to = None if in_place else (pages + torch.randperm(300, generator=g, device="cuda")[:282]).int().view(1, 282)
    batch = c.CachedRows(torch.zeros(2, **i32), torch.tensor([length], **i32), table)
    kept, left = c.cached_evict(c.PagedCache(pool), batch, weights, keep, first, recent, table_out=to)
    assert torch.equal(kept[0].long(), want) and int(left) == keep
    new = torch.where(given[0].isnan(), 99.0, given[0])
    now = torch.where(weights[0].isnan(), 99.0, weights[0])
    assert torch.equal(now[:, :keep], new.gather(1, want)) and not bool(now[:, keep:length].any()) and torch.equal(now[:, length:], new[:, length:])
    slot, there = torch.arange(keep, device="cuda"), (table if to is None else to)[0].long()
    for h in range(nkv):
        for which in range(2):
            x = start[table[0].long()[want[h] // page], 0, which, h, want[h] % page]
            assert torch.equal(pool[there[slot // page], 0, which, h, slot % page], x)


FIRST_CALLS = """
import torch
from paper_2603_09215_amd import cached as c
g = torch.Generator(device="cuda").manual_seed(65)
m, pages = 2600, 41
pool = torch.randn(pages, 1, 2, 4, 64, 128, generator=g, device="cuda").bfloat16()
new = [torch.randn(m, h, 128, generator=g, device="cuda").bfloat16() for h in (28, 4, 4)]
i32 = dict(dtype=torch.int32, device="cuda")
cache, batch = c.PagedCache(pool), c.CachedRows(torch.tensor([0, m], **i32), torch.tensor([m], **i32), torch.randperm(pages, generator=g, device="cuda").int().view(1, pages))
turn = c.Rotation(128)
def calls():
    lse = torch.empty(m, 28, device="cuda")
    q = c.cached_append(*new, cache, batch, rotation=turn)
    out = c.cached_attend(q, cache, batch, lse=lse)
    weights = c.cached_weigh(q, lse, cache, batch)
    kept, left = c.cached_evict(cache, batch, weights, 1000, 4, 32, weights_out=torch.zeros_like(weights))
    return q, out, lse, weights, kept, left
torch.cuda.synchronize()
graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph):
    captured = calls()
for turn_of in range(3):
    for t in captured:
        t.fill_(3)
    graph.replay()
    torch.cuda.synchronize()
    got = [t.clone() for t in captured]
    eager = calls()
    torch.cuda.synchronize()
    for x, y in zip(got, eager):
        assert torch.equal(x, y), turn_of
print("as eager calls")
"""


def test_first_calls_of_a_process_captured():
    """kernels that ask for more LDS than 64 KiB among them"""
    gpu()
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, "-c", FIRST_CALLS], cwd=root, capture_output=True, text=True, timeout=100)
    assert r.returncode == 0 and "as eager calls" in r.stdout, r.stderr[-2000:]
