"""The operators on a paged cache with operands of one row, whose stride torch may say anything of: on the CPU, with tensors that say they are on a GPU."""
import pytest
import torch

from paper_2603_09215_amd import SparkError, cached
from test_cached_tensors import BF16, F32, I32, on


class Reached(Exception):
    pass


@pytest.fixture()
def strides(monkeypatch):
    """the strides that a call would be launched with"""
    seen = []

    def launch(what, tensors, written, call, *args):
        seen.extend(args)
        raise Reached
    monkeypatch.setattr(cached, "_launch", launch)
    monkeypatch.setattr(cached, "attend_workspace_bytes", lambda *a: 0)
    return seen


def one_row(heads, dtype=BF16, width=5 * 64 + 3):
    """a row of a matrix whose rows are not apart by a multiple of eight elements"""
    return on(9, width, dtype=dtype)[:, :heads * 64].unflatten(1, (heads, 64))[8:9]   # (its address is a multiple of 16 bytes)


def batch(c):
    return c, cached.CachedRows(on(2, dtype=I32), on(1, dtype=I32), on(1, 2, dtype=I32))


def test_a_row_of_any_matrix(strides):
    c, b = batch(cached.PagedCache(on(4, 2, 2, 2, 16, 64)))
    q, k = one_row(4), one_row(2)
    assert q.stride(0) % 8
    lse, given = on(1, 4, dtype=F32), one_row(4)
    for call, want in ((lambda: cached.cached_attend(q, c, b, out=given), [256, 256]), (lambda: cached.cached_weigh(q, lse, c, b, out=on(1, 2, 32, dtype=F32)), [256]),
                       (lambda: cached.cached_append(q, k, k, c, b, out=given), [256, 128, 128, 256])):
        strides.clear()
        with pytest.raises(Reached):
            call()
        assert [x for x in strides if x in (256, 128, 323)] == want
    for rows in (on(3, 323)[:2, :256].unflatten(1, (4, 64)), on(1, 4, 64).expand(2, 4, 64)):   # (two rows: apart, and by multiples)
        with pytest.raises(SparkError):
            cached.cached_attend(rows, c, b)


def test_an_expanded_row(strides):
    c, b = batch(cached.PagedCache(on(4, 2, 2, 2, 16, 64)))
    q = on(4, 64).expand(1, 4, 64)
    with pytest.raises(Reached):
        cached.cached_attend(q, c, b, out=on(1, 4, 64))
    assert strides.count(256) == 2
