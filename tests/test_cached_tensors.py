"""What paper_2603_09215_amd/cached.py refuses before it reaches the library or the GPU: on the CPU, with tensors that say they are
on a GPU."""
import math

import pytest
import torch

from paper_2603_09215_amd import SparkError, cached

F32, BF16, I32 = torch.float32, torch.bfloat16, torch.int32


class OnGpu(torch.Tensor):
    is_cuda = True

    def get_device(self):
        raise AssertionError("reached the launch")


def on(*shape, dtype=BF16):
    return torch.zeros(*shape, dtype=dtype).as_subclass(OnGpu)


@pytest.fixture()
def it():
    c = cached.PagedCache(on(4, 2, 2, 2, 16, 64))
    b = cached.CachedRows(on(3, dtype=I32), on(2, dtype=I32), on(2, 2, dtype=I32))
    return c, b, on(3, 4, 64), on(3, 2, 64), on(3, 2, 64)


def refused(call, match=None):
    with pytest.raises(SparkError, match=match):
        call()


def test_pools():
    for pool in (torch.zeros(4, 1, 2, 2, 16, 64), on(4, 2, 2, 16, 64), on(4, 1, 3, 2, 16, 64), on(4, 1, 2, 2, 24, 64), on(4, 1, 2, 2, 16, 96), on(0, 1, 2, 2, 16, 64),
                 on(4, 1, 2, 0, 16, 64), on(4, 1, 2, 2, 16, 64, dtype=torch.float16), on(4, 1, 2, 2, 64, 16).transpose(4, 5), "pool"):
        refused(lambda: cached.PagedCache(pool))


def test_batches():
    good = [on(3, dtype=I32), on(2, dtype=I32), on(2, 2, dtype=I32)]
    for at, bad in ((0, torch.zeros(3, dtype=I32)), (0, on(2, dtype=I32)), (0, on(3, dtype=torch.int64)), (1, on(3, dtype=I32)), (1, on(4, dtype=I32)[::2]),
                    (2, on(4, dtype=I32)), (2, on(3, 2, dtype=I32)), (2, on(2, 0, dtype=I32)), (2, None)):
        args = list(good)
        args[at] = bad
        refused(lambda: cached.CachedRows(*args))


def test_rotations():
    for kw in (dict(rotary=3), dict(rotary=-2), dict(rotary=130), dict(rotary=64, base=0.0), dict(rotary=64, factor=0.0), dict(rotary=64, original=0),
               dict(rotary=64, low=4.0, high=1.0), dict(rotary=64, amplitude=math.inf), dict(rotary=64, freqs=[1.0] * 31)):
        refused(lambda: cached.Rotation(device="cpu", **kw))


def test_frequencies():
    """as the formula says, at waves of many turns, few, and between; a step; and all of them"""
    plain = cached.Rotation(64, device="cpu").freqs
    assert torch.allclose(plain, 10000.0 ** (-torch.arange(0, 64, 2, dtype=torch.float64) / 64), rtol=1e-14, atol=0)
    f = cached.Rotation(64, factor=8.0, low=1.0, high=4.0, original=8192, device="cpu").freqs
    turns = 8192 * plain / (2 * math.pi)
    assert torch.equal(f[turns >= 4], plain[turns >= 4]) and torch.equal(f[turns <= 1], plain[turns <= 1] / 8)
    mid = (turns > 1) & (turns < 4)
    share = (turns[mid] - 1) / 3
    assert bool(mid.any()) and torch.allclose(f[mid], plain[mid] * (share + (1 - share) / 8), rtol=1e-12, atol=0)
    step = cached.Rotation(64, factor=8.0, low=2.0, high=2.0, device="cpu").freqs
    assert torch.equal(step, torch.where(turns >= 2, plain, plain / 8))
    every = cached.Rotation(64, factor=4.0, low=math.inf, high=math.inf, device="cpu").freqs
    assert torch.equal(every, plain / 4)
    assert torch.equal(cached.Rotation(4, freqs=[0.5, 0.25], device="cpu").freqs, torch.tensor([0.5, 0.25], dtype=torch.float64))
    assert cached.Rotation(0, device="cpu").freqs.shape == (0,)


def test_append(it):
    c, b, q, k, v = it
    for kw in (dict(q=torch.zeros(3, 4, 64)), dict(q=on(3, 4, 32)), dict(q=on(3, 256)), dict(q=on(3, 3, 64)), dict(q=on(3, 4, 64, dtype=torch.float16)),
               dict(k=on(3, 4, 64)), dict(k=on(2, 2, 64)), dict(k=on(3, 2, 64, dtype=F32)), dict(v=on(3, 1, 64)), dict(v=on(3, 64, 2).transpose(1, 2)),
               dict(out=on(3, 4, 64, dtype=F32)), dict(out=on(2, 4, 64)), dict(positions=on(3, dtype=torch.int64)), dict(positions=on(2, dtype=I32)),
               dict(q_gain=on(64)), dict(k_gain=on(32, dtype=F32)), dict(eps=-1.0), dict(eps=math.nan), dict(rotation=cached.Rotation(128, device="cpu")), dict(layer=2),
               dict(layer=-1)):
        a = dict(q=q, k=k, v=v, cache=c, batch=b)
        refused(lambda: cached.cached_append(**{**a, **kw}))


def test_attend_and_weigh(it):
    c, b, q, _, _ = it
    wide = on(3, 4 * 64 + 4)[:, :256].unflatten(1, (4, 64))
    for kw in (dict(q=on(3, 4, 64, dtype=F32)), dict(q=on(3, 3, 64)), dict(q=wide), dict(q=on(3, 8, 64)[:, ::2]), dict(out=on(3, 4, 64, dtype=F32)), dict(out=wide),
               dict(out=on(3, 2, 64)), dict(lse=on(3, 4)), dict(lse=on(4, 3, dtype=F32)), dict(scale=0.0), dict(scale=math.nan), dict(scale=1e300), dict(scale=1e-300),
               dict(layer=2)):
        refused(lambda: cached.cached_attend(**{**dict(q=q, cache=c, batch=b), **kw}))
    good = dict(q=q, lse=on(3, 4, dtype=F32), cache=c, batch=b)
    for kw in (dict(q=wide), dict(lse=on(3, 2, dtype=F32)), dict(lse=None), dict(before=on(2, 2, 31, dtype=F32)), dict(before=on(2, 2, 32)), dict(out=on(2, 2, 16, dtype=F32)),
               dict(decay=math.inf), dict(decay=1e300), dict(scale=0.0), dict(layer=3)):
        refused(lambda: cached.cached_weigh(**{**good, **kw}))


def test_evict(it):
    c, b, _, _, _ = it
    w = on(2, 2, 32, dtype=F32)
    for kw in (dict(keep=0), dict(keep=33), dict(keep=4, first=3, recent=2), dict(keep=4, first=-1), dict(keep=4, recent=-1), dict(weights=on(2, 2, 32)),
               dict(weights=on(2, 1, 32, dtype=F32)), dict(weights_out=on(2, 2, 31, dtype=F32)), dict(table_out=on(2, 1, dtype=torch.int64)), dict(table_out=on(1, 1, dtype=I32)),
               dict(keep=17, table_out=on(2, 1, dtype=I32))):
        refused(lambda: cached.cached_evict(**{**dict(cache=c, batch=b, weights=w, keep=16), **kw}))
    refused(lambda: cached.cached_evict(c, b, w, 16, table_out=b.table.view(-1)[:2].view(2, 1)), "a part of")
    for scale in (0.0, 1e-50, 3e38, math.inf, math.nan):
        refused(lambda: cached._scale(scale, 64), "scale")
    assert cached._scale(None, 64) == 0.125 and cached._scale(-2.0 ** 127, 64) == -2.0 ** 127


def test_sizes_past_the_calls_limits():
    c = cached.PagedCache(on(4, 2, 2, 2, 16, 64))
    b = object.__new__(cached.CachedRows)
    for m, pages, n in (((1 << 22) + 1, 4, 2), (3, (1 << 20) + 1, 2), (3, 4, (1 << 19) + 1)):
        b.n, b.max_pages = n, pages
        refused(lambda: b._of(m, c), "are taken")
    refused(lambda: cached.cached_append(on(3, 6, 64), on(3, 4, 64), on(3, 4, 64), cached.PagedCache(on(4, 2, 2, 4, 16, 64)), b), "a multiple")
    refused(lambda: cached._group((1 << 14) + 1, 1 << 12, c), "2\\^26")
