"""Attention over a bf16 cache: how many bits of the probabilities reach the product with the values.  Queries of four channels, so that scores
are off by a few last bits of fp32, and rows that see few slots, so that sums are: what remains is the result's own rounding, and the probabilities'."""
import pytest
import torch

import cached_ref as ref
from test_gpu_cached import gpu, make_batch, near, rows_of
from test_gpu_cached_long import full_pool

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16
CHANNELS, SCALE = 4, 0.5

# (rows, length), pages of a sequence's table, query heads, kv heads, head_dim: streams and both tiles, in one part and in several
KINDS = [([(1, 64)], 4, 28, 4, 128), ([(1, 70), (1, 40)], 5, 4, 2, 64), ([(1, 200)], 188, 7, 1, 128), ([(3, 150)], 125, 8, 2, 64),
         ([(900, 901)], 57, 14, 2, 64), ([(3500, 3500)], 55, 32, 2, 64), ([(300, 320)], 63, 28, 4, 128), ([(500, 500), (400, 450)], 8, 28, 4, 128),
         ([(700, 720)], 40, 28, 4, 128), ([(2500, 2600)], 41, 28, 4, 128)]


@pytest.mark.parametrize("shape,table_pages,nq,nkv,hd", KINDS)
def test_probabilities_have_sixteen_bits(shape, table_pages, nq, nkv, hd):
    c, page = gpu(), 64
    starts, lengths, table, pages, m = make_batch(shape, page, 91, max_pages=table_pages)
    b = ref.Batch(starts, lengths, table, m, pages, page)
    pool, q = full_pool(pages, 1, nkv, page, hd, BF16, 92), rows_of(m, nq, hd, BF16, 93)
    q[:, :, CHANNELS:] = 0.0
    got = c.cached_attend(q, c.PagedCache(pool), c.CachedRows(starts.cuda(), lengths.cuda(), table.cuda()), scale=SCALE)
    u, group, few = ref.U, nq // nkv, 200
    # an output: half a step of bf16; a probability: two parts of bf16, each rounded to half a step of what it has to hold
    step, parts = ref.half_step(BF16), ref.half_step(BF16) ** 2
    would_be_seen = False
    for s in range(b.n):
        first = b.length[s] - b.rows[s]
        rows = torch.arange(b.rows[s], device="cuda")
        rows = rows[first + rows < few]           # (rows that see few slots)
        assert rows.numel()
        slot = torch.arange(few, device="cuda").clamp(max=b.length[s] - 1)
        at = torch.tensor(b.table[s], device="cuda")[slot // page].long()
        sees = torch.arange(few, device="cuda")[None] <= (first + rows)[:, None]
        for h in range(nq):
            k, v = (pool[at, 0, w, h // group, slot % page].double() for w in (0, 1))
            x = q[b.row0[s] + rows, h].double()
            score = (x @ k.t().contiguous() * SCALE).masked_fill(~sees, -torch.inf)
            off = (x.abs() @ k.abs().t().contiguous() * SCALE * (CHANNELS + 3) * u).masked_fill(~sees, 0.0)
            top = score.amax(1, keepdim=True)
            p = torch.exp(score - top)
            share = p / p.sum(1, keepdim=True)
            n = sees.sum(1, keepdim=True)
            # of a probability: its score and the maximum, the exponent's rounding and the exponential's steps (as in cached_ref.attend)
            each = off + off.amax(1, keepdim=True) + (4 + 2 * torch.where(sees, top - score, 0.0)) * 2 * u
            want, mags = share @ v, share @ v.abs()
            tol = (share * each) @ v.abs() + mags * ((share * each).sum(1, keepdim=True) + 4 * (n + 16) * u + parts) + step * want.abs()
            near(got[b.row0[s] + rows, h], want.cpu(), tol.cpu(), f"head {h}")
            once = (p.to(BF16).double() @ v) / p.sum(1, keepdim=True)   # the same with probabilities of one part
            would_be_seen |= bool(((once.to(BF16).double() - want).abs() > tol).any())
    assert would_be_seen
