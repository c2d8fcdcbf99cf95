"""The operators on a paged cache against their formulas in 64 bits (tests/cached_ref.py)."""
import math

import pytest
import torch

import cached_ref as ref

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16


def gpu():
    from paper_2603_09215_amd import cached
    return cached


def make_batch(shape, page, seed, max_pages=None, spare=3, before=0, behind=0, holes=()):
    """(starts, lengths, table, pages in the pool, rows): `shape` (rows, length) of each sequence, pages in any order; `before` and
    `behind`: rows that are nobody's; holes: (sequence, page) without a page"""
    g = torch.Generator().manual_seed(seed)
    n = len(shape)
    max_pages = max_pages or max(1, max(-(-c // page) for _, c in shape))
    total = n * max_pages + spare
    table = torch.randperm(total, generator=g)[:n * max_pages].view(n, max_pages).int()
    for s, p in holes:
        table[s, p] = -1 if (s + p) % 2 else total
    starts = [before]
    for r, _ in shape:
        starts.append(starts[-1] + r)
    return torch.tensor(starts, dtype=torch.int32), torch.tensor([c for _, c in shape], dtype=torch.int32), table, total, starts[-1] + behind


def near(got, want, tol, what):
    """within tol where `want` is a number"""
    got, there = got.double().cpu(), ~want.isnan()
    assert bool(torch.isfinite(got[there & torch.isfinite(want)]).all()), what
    inf = there & torch.isinf(want)
    assert torch.equal(got[inf], want[inf]), what
    there &= ~inf
    worst = ((got - want).abs() - tol)[there]
    assert worst.numel() == 0 or float(worst.max()) <= 0, f"{what}: {float(worst.max())} past the tolerance"


def same(a, b):
    """bit by bit"""
    return torch.equal(a.contiguous().view(torch.uint8), b.contiguous().view(torch.uint8))


SHAPES = {
    "one": ([(1, 1)], 16),
    "step": ([(1, 130)], 64),
    "chunk": ([(37, 37)], 16),
    "ragged": ([(3, 77), (1, 1), (0, 40), (20, 20), (5, 3), (2, 0), (18, 129)], 48),   # (rows without a slot, a sequence without any)
}


def rows_of(m, heads, hd, dtype, seed, kind="plain"):
    g = torch.Generator().manual_seed(seed)
    if kind == "plain":
        return torch.randn(m, heads, hd, generator=g).to(dtype).cuda()
    whole = torch.randn(m, heads * hd + 24, generator=g).to(dtype).cuda()   # views of wider rows
    return whole[:, 8:8 + heads * hd].unflatten(1, (heads, hd)) if kind == "wide" else whole[:, 3:3 + heads * hd].unflatten(1, (heads, hd))


@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("nq,nkv,hd,dtype,src,rotary,interleaved,norm,kind", [
    (4, 2, 64, BF16, F32, 64, False, False, "plain"), (7, 1, 128, BF16, BF16, 128, False, True, "wide"), (6, 3, 64, F32, F32, 24, True, True, "odd"),
    (4, 4, 128, F32, BF16, 64, True, False, "wide"), (2, 1, 64, BF16, BF16, 10, False, True, "plain"), (3, 1, 128, BF16, F32, 0, False, True, "plain"),
    (2, 2, 128, F32, F32, 128, True, True, "plain"), (5, 1, 64, BF16, F32, 6, True, False, "odd")])
def test_append(shape, nq, nkv, hd, dtype, src, rotary, interleaved, norm, kind):
    c = gpu()
    shape, page = SHAPES[shape]
    starts, lengths, table, pages, m = make_batch(shape, page, 1, before=2, behind=3, holes=[(0, 0)] if len(shape) > 2 else [])
    b = ref.Batch(starts, lengths, table, m, pages, page)
    pool = torch.randn(pages, 2, 2, nkv, page, hd).to(dtype)
    q, k, v = (rows_of(m, h, hd, src, 5 + i, kind) for i, h in enumerate((nq, nkv, nkv)))
    gains = [1 + 0.1 * torch.randn(hd) if norm else None for _ in range(2)]
    positions = torch.randint(-5, 200000, (m,)).int() if norm else None
    amplitude = 1.25 if rotary == 24 else 1.0
    turn = c.Rotation(rotary, interleaved=interleaved, amplitude=amplitude)
    cache = c.PagedCache(pool.cuda())
    out = torch.full((m, nq, hd), 7.0, dtype=dtype, device="cuda")
    got = c.cached_append(q, k, v, cache, c.CachedRows(starts.cuda(), lengths.cuda(), table.cuda()), layer=1, rotation=turn,
                          q_gain=None if gains[0] is None else gains[0].cuda(), k_gain=None if gains[1] is None else gains[1].cuda(), eps=1e-5,
                          positions=None if positions is None else positions.cuda(), out=out)
    assert got is out
    want, tol, new, new_tol = ref.append(q.cpu(), k.cpu(), v.cpu(), pool, b, 1, rotary, interleaved, ref.frequencies(rotary), amplitude, *gains, 1e-5, positions)
    near(out, want, tol, "q")
    assert bool((out.cpu()[want.isnan()] == 7).all())
    near(cache.pool, new, new_tol, "pool")
    untouched = new == pool.double()
    assert bool((cache.pool.cpu()[untouched] == pool[untouched]).all())


def test_append_in_place_and_far_positions():
    c = gpu()
    starts, lengths, table, pages, m = make_batch([(9, 9)], 16, 2)
    q, k, v = (rows_of(m, h, 64, F32, 3 + i) for i, h in enumerate((4, 2, 2)))
    positions = torch.tensor([0, 1, -1, 12345, 999999, 16777217, 2 ** 31 - 1, -2 ** 31, 8191], dtype=torch.int32)
    pool = torch.zeros(pages, 1, 2, 2, 16, 64)
    b = ref.Batch(starts, lengths, table, m, pages, 16)
    want, tol, new, new_tol = ref.append(q.cpu(), k.cpu(), v.cpu(), pool, b, 0, 64, False, ref.frequencies(64), positions=positions)
    cache = c.PagedCache(pool.cuda())
    batch = c.CachedRows(starts.cuda(), lengths.cuda(), table.cuda())
    got = c.cached_append(q, k, v, cache, batch, rotation=c.Rotation(64), positions=positions.cuda(), out=q)
    assert got is q
    near(q, want, tol, "q")
    near(cache.pool, new, new_tol, "pool")


@pytest.mark.parametrize("size", [1e-30, 1e25])
def test_append_norms_outside_fp32s_squares(size):
    c = gpu()
    starts, lengths, table, pages, m = make_batch([(3, 3)], 16, 2)
    q, k, v = (rows_of(m, h, 64, F32, 3 + i) * size for i, h in enumerate((2, 1, 1)))
    gain = torch.ones(64)
    b = ref.Batch(starts, lengths, table, m, pages, 16)
    pool = torch.zeros(pages, 1, 2, 1, 16, 64)
    want, tol, new, new_tol = ref.append(q.cpu(), k.cpu(), v.cpu(), pool, b, 0, q_gain=gain, k_gain=gain, eps=0.0)
    cache = c.PagedCache(pool.cuda())
    got = c.cached_append(q, k, v, cache, c.CachedRows(starts.cuda(), lengths.cuda(), table.cuda()), q_gain=gain.cuda(), k_gain=gain.cuda(), eps=0.0)
    near(got, want, tol, "q")
    near(cache.pool, new, new_tol, "pool")


def attend_case(shape, page, nq, nkv, hd, dtype, seed, causal=True, scale=None, kind="plain", holes=(), layers=1, before=1, behind=2, rubbish=True, std=1.0):
    """runs it and compares out and lse; the slots behind the lengths and pages of nobody hold NaN and infinities"""
    c = gpu()
    starts, lengths, table, pages, m = make_batch(shape, page, seed, before=before, behind=behind, holes=holes)
    b = ref.Batch(starts, lengths, table, m, pages, page)
    g = torch.Generator().manual_seed(seed)
    pool = torch.full((pages, layers, 2, nkv, page, hd), math.nan)
    pool[..., ::3] = math.inf
    if not rubbish:
        pool.zero_()
    for s in range(b.n):
        for t in range(b.length[s]):
            if b.page(s, t) is not None:
                pool[b.page(s, t), layers - 1, :, :, t % page] = torch.randn(2, nkv, hd, generator=g)
    pool = pool.to(dtype)
    q = (rows_of(m, nq, hd, dtype, seed + 1, kind) * std).to(dtype)
    if kind == "wide":
        q = rows_of(m, nq, hd, dtype, seed + 1, kind)
    cache, batch = c.PagedCache(pool.cuda()), c.CachedRows(starts.cuda(), lengths.cuda(), table.cuda())
    out, lse = torch.full((m, nq, hd), 7.0, dtype=dtype, device="cuda"), torch.full((m, nq), 7.0, device="cuda")
    assert c.cached_attend(q, cache, batch, layer=layers - 1, scale=scale, causal=causal, out=out, lse=lse) is out
    want, tol, want_lse, lse_tol = ref.attend(q.cpu(), pool, b, layers - 1, hd ** -0.5 if scale is None else scale, causal)
    near(lse, want_lse, lse_tol, "lse")
    near(out, want, tol, "out")
    nobody = want_lse.isnan()
    assert bool((out.cpu()[nobody] == 7).all()) and bool((lse.cpu()[nobody] == 7).all())
    again, again_lse = torch.empty_like(out), torch.empty_like(lse)
    c.cached_attend(q, cache, batch, layer=layers - 1, scale=scale, causal=causal, out=again, lse=again_lse)
    there = ~nobody
    assert same(again.cpu()[there], out.cpu()[there]) and same(again_lse.cpu()[there], lse.cpu()[there])
    return c, cache, batch, b, q, out, lse


HEADS = [(4, 2, 64), (7, 1, 128), (16, 1, 64), (24, 1, 128), (3, 3, 128)]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("nq,nkv,hd", HEADS)
@pytest.mark.parametrize("shape", SHAPES)
def test_attend(shape, nq, nkv, hd, dtype):
    shape, page = SHAPES[shape]
    attend_case(shape, page, nq, nkv, hd, dtype, 11)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("rows", [1, 2, 3, 5, 9, 33, 64, 65])
@pytest.mark.parametrize("length", [65, 300])
def test_attend_rows(rows, length, dtype):
    attend_case([(rows, length)], 32, 7, 1, 128, dtype, 12)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("shape,page", [([(3, 77), (0, 40), (1, 1), (40, 21)], 16), ([(50, 130)], 80)])
def test_attend_all_slots_strides_layers_and_scales(shape, page, dtype):
    attend_case(shape, page, 6, 2, 64, dtype, 13, causal=False, layers=3, kind="wide")
    attend_case(shape, page, 6, 2, 64, dtype, 14, scale=-0.3, kind="wide")
    attend_case(shape, page, 6, 2, 64, dtype, 15, scale=0.7, std=4.0)   # next to one-hot


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_attend_pages_that_are_none(dtype):
    """a hole at the start, in the middle and over a whole tile, a sequence of nothing but holes"""
    shape = [(4, 200), (20, 150), (2, 30), (1, 16)]
    attend_case(shape, 16, 4, 2, 64, dtype, 16, holes=[(0, 0), (0, 5), (0, 6), (0, 7), (0, 8), (0, 9), (1, 9), (2, 0), (2, 1), (3, 0)])


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("rows", [1, 6, 130])
def test_no_number_reaches_rows_that_do_not_see_it(rows, dtype):
    """a NaN and infinities in the new rows' own keys and values: the rows before them give what they give without, and an infinite value that is seen
    its infinity"""
    c = gpu()
    nq, nkv, hd, page, length = 7, 1, 128, 32, 150 + rows
    starts, lengths, table, pages, m = make_batch([(rows, length)], page, 3)
    pool = torch.randn(pages, 1, 2, nkv, page, hd).to(dtype)
    q = rows_of(m, nq, hd, dtype, 4)
    batch = c.CachedRows(starts.cuda(), lengths.cuda(), table.cuda())
    clean = c.cached_attend(q, c.PagedCache(pool.cuda()), batch)
    b = ref.Batch(starts, lengths, table, m, pages, page)
    row = rows // 2   # from this row on it is seen
    slot = b.slot(0, row)
    for which, value in ((1, math.inf), (1, -math.inf), (1, math.nan), (0, math.nan), (0, math.inf)):
        bad = pool.clone()
        bad[b.page(0, slot), 0, which, 0, slot % page, 5] = value
        got = c.cached_attend(q, c.PagedCache(bad.cuda()), batch)
        assert same(got[:row], clean[:row]), (which, value)
        if which == 1:
            hit = got[row:, :, 5].float()
            assert bool(hit.isnan().all()) if math.isnan(value) else bool((hit == value).all()), value
            rest = torch.arange(hd) != 5
            assert bool(torch.isfinite(got[row:][:, :, rest.cuda()]).all())
        elif math.isnan(value):
            assert bool(got[row:].isnan().all())


def weigh_case(shape, page, nq, nkv, hd, dtype, seed, causal=True, before=True, decay=0.75, in_place=False, holes=()):
    c, cache, batch, b, q, out, lse = attend_case(shape, page, nq, nkv, hd, dtype, seed, causal=causal, holes=holes)
    prior = torch.rand(b.n, nkv, b.slots, device="cuda") if before else None
    result = prior.clone() if in_place else torch.full((b.n, nkv, b.slots), 7.0, device="cuda")
    got = c.cached_weigh(q, lse, cache, batch, causal=causal, before=result if in_place else prior, decay=decay, out=result)
    assert got is result
    want, tol = ref.weigh(q.cpu(), lse.cpu(), cache.pool.cpu(), b, 0, hd ** -0.5, None if prior is None else prior.cpu(), decay, causal)
    near(result, want, tol, "weights")
    rest = want.isnan()
    assert torch.equal(result.cpu()[rest], prior.cpu()[rest] if in_place else torch.full_like(result.cpu(), 7.0)[rest])
    if not in_place:
        again = c.cached_weigh(q, lse, cache, batch, causal=causal, before=prior, decay=decay)
        assert same(again.cpu()[~rest], result.cpu()[~rest]) and bool((again.cpu()[rest] == 0).all())


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("nq,nkv,hd", HEADS)
@pytest.mark.parametrize("shape", SHAPES)
def test_weigh(shape, nq, nkv, hd, dtype):
    shape, page = SHAPES[shape]
    weigh_case(shape, page, nq, nkv, hd, dtype, 21)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_weigh_kinds(dtype):
    weigh_case([(70, 200), (1, 9)], 80, 4, 2, 64, dtype, 22, causal=False, before=False)
    weigh_case([(70, 200), (1, 9)], 16, 4, 2, 64, dtype, 23, in_place=True, holes=[(0, 3), (1, 0)])
    weigh_case([(33, 64)], 32, 4, 2, 64, dtype, 24, decay=0.0)


def test_weigh_without_rows():
    c = gpu()
    starts, lengths, table, pages, m = make_batch([(0, 20), (0, 0)], 16, 2)
    cache, batch = c.PagedCache.empty(pages, 2, 64, 16), c.CachedRows(starts.cuda(), lengths.cuda(), table.cuda())
    before = torch.rand(2, 2, 32, device="cuda")
    out = c.cached_weigh(torch.empty(0, 4, 64, dtype=BF16, device="cuda"), torch.empty(0, 4, device="cuda"), cache, batch, before=before, decay=0.5)
    assert torch.equal(out[0, :, :20], 0.5 * before[0, :, :20]) and not bool(out[0, :, 20:].any()) and not bool(out[1].any())


KINDS = ["plain", "ties", "zeros", "odd"]


def some_weights(n, nkv, slots, kind, seed):
    g = torch.Generator().manual_seed(seed)
    w = torch.exp(2 * torch.randn(n, nkv, slots, generator=g))
    if kind == "ties":
        w = torch.randint(0, 3, (n, nkv, slots), generator=g).float()
    elif kind == "zeros":
        w = torch.where(torch.rand(n, nkv, slots, generator=g) < 0.5, 0.0, -0.0)
    elif kind == "odd":   # anything that fp32 holds
        w = torch.randn(n, nkv, slots, generator=g) * 10.0 ** torch.randint(-44, 38, (n, nkv, slots), generator=g).double()
        w = w.float()
        for value in (math.inf, -math.inf, math.nan, -0.0, 0.0):
            w[torch.rand(n, nkv, slots, generator=g) < 0.05] = value
    return w


@pytest.mark.parametrize("in_place", [True, False])
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("shape,page,keep,first,recent", [
    ([(1, 1)], 16, 1, 0, 0), ([(1, 40), (1, 17), (1, 16), (1, 0), (1, 5)], 16, 16, 2, 3), ([(1, 3000), (1, 2500)], 48, 1025, 4, 32),
    ([(1, 300)], 64, 36, 4, 32), ([(1, 130)], 16, 128, 0, 128), ([(1, 130)], 16, 1, 1, 0), ([(1, 2100)], 32, 2099, 0, 0)])
def test_evict(shape, page, keep, first, recent, kind, in_place):
    c = gpu()
    nkv, hd, dtype = (2, 128, BF16) if page != 16 else (3, 64, F32)
    _, lengths, table, pages, _ = make_batch(shape, page, 5)
    n, max_pages = table.shape
    out_pages = -(-keep // page)
    table_out = None if in_place else (pages + torch.randperm(n * out_pages + 1)[:n * out_pages]).view(n, out_pages).int()
    total = pages + (0 if in_place else n * out_pages + 1)
    pool = torch.randn(total, 2, 2, nkv, page, hd).to(dtype)
    w = some_weights(n, nkv, max_pages * page, kind, 6)
    b = ref.Batch([0] * (n + 1), lengths, table, 0, total, page)
    want_pool, want_kept, want_lengths, want_w, touched = ref.evict(pool, b, 1, w, keep, first, recent, table_out)
    cache, batch = c.PagedCache(pool.cuda()), c.CachedRows(torch.zeros(n + 1, dtype=torch.int32, device="cuda"), lengths.cuda(), table.cuda())
    weights = w.cuda()
    weights_out = None if in_place else torch.full_like(weights, 7.0)
    kept, new_lengths = c.cached_evict(cache, batch, weights, keep, first, recent, layer=1, table_out=None if in_place else table_out.cuda(), weights_out=weights_out)
    assert torch.equal(kept.cpu(), want_kept) and torch.equal(new_lengths.cpu(), want_lengths)
    assert same(cache.pool.cpu(), want_pool)
    got_w = (weights if in_place else weights_out).cpu()
    assert same(got_w[touched], want_w[touched])
    assert same(got_w[~touched], (w if in_place else torch.full_like(w, 7.0))[~touched])
    if not in_place:
        assert same(weights.cpu(), w)


def test_evict_pages_that_are_none():
    c = gpu()
    _, lengths, table, pages, _ = make_batch([(1, 100), (1, 64)], 16, 7, holes=[(0, 1), (0, 3), (1, 0)])
    pool, w = torch.randn(pages, 1, 2, 2, 16, 64), some_weights(2, 2, table.shape[1] * 16, "plain", 8)
    b = ref.Batch([0] * 3, lengths, table, 0, pages, 16)
    want_pool, want_kept, want_lengths, _, _ = ref.evict(pool, b, 0, w, 50, 1, 7)
    cache = c.PagedCache(pool.cuda())
    kept, new = c.cached_evict(cache, c.CachedRows(torch.zeros(3, dtype=torch.int32, device="cuda"), lengths.cuda(), table.cuda()), w.cuda(), 50, 1, 7)
    assert torch.equal(kept.cpu(), want_kept) and torch.equal(new.cpu(), want_lengths) and same(cache.pool.cpu(), want_pool)


def test_what_starts_and_lengths_may_hold():
    """starts that go down and past the rows, lengths below zero and past the pages: cut to their ranges"""
    c = gpu()
    nq, nkv, hd, page, m = 4, 2, 64, 16, 9
    starts, lengths = torch.tensor([-3, 4, 2, 400], dtype=torch.int32), torch.tensor([1000, -5, 40], dtype=torch.int32)
    table = torch.arange(9).view(3, 3).int()
    b = ref.Batch(starts, lengths, table, m, 9, page)
    pool = torch.randn(9, 1, 2, nkv, page, hd)
    cache, batch = c.PagedCache(pool.cuda()), c.CachedRows(starts.cuda(), lengths.cuda(), table.cuda())
    q, k, v = (rows_of(m, h, hd, F32, 31 + i) for i, h in enumerate((nq, nkv, nkv)))
    out = torch.full_like(q, 7.0)
    c.cached_append(q, k, v, cache, batch, out=out)
    # (rows 2 and 3 are asked for by two sequences: of their results nothing is said)
    assert torch.equal(out[[0, 1, 4, 5, 6, 7, 8]], q[[0, 1, 4, 5, 6, 7, 8]])
    lse = torch.empty(m, nq, device="cuda")
    got = c.cached_attend(q, cache, batch, lse=lse)
    want, tol, _, _ = ref.attend(q.cpu(), cache.pool.cpu(), b, 0, hd ** -0.5)
    clear = [0, 1, 4, 5, 6, 7, 8]
    near(got[clear], want[clear], tol[clear], "out")
    c.cached_weigh(q, lse, cache, batch)
    c.cached_evict(cache, batch, torch.rand(3, nkv, 48, device="cuda"), 8)
    torch.cuda.synchronize()
