"""That a refused gradient names the operator that has none, of those on a paged cache as of those on 8-bit rows: on the CPU, with tensors that say they are on
a GPU."""
import pytest
import torch

from paper_2603_09215_amd import SparkError, cached, scaled


class On(torch.Tensor):
    is_cuda = True

    def get_device(self):
        return 0


def on(*shape, dtype=torch.bfloat16):
    return torch.zeros(*shape, dtype=dtype).as_subclass(On)


def test_the_operator_is_named(monkeypatch):
    monkeypatch.setattr(cached, "attend_workspace_bytes", lambda *a: 0)
    c, b = cached.PagedCache(on(4, 1, 2, 2, 16, 64)), cached.CachedRows(on(3, dtype=torch.int32), on(2, dtype=torch.int32), on(2, 2, dtype=torch.int32))
    q, k, out = on(3, 4, 64).requires_grad_(), on(3, 2, 64), on(3, 4, 64)
    lse, w = on(3, 4, dtype=torch.float32), on(2, 2, 32, dtype=torch.float32)
    for name, call in (("cached_append", lambda: cached.cached_append(q, k, k, c, b, out=out)), ("cached_attend", lambda: cached.cached_attend(q, c, b, out=out)),
                       ("cached_weigh", lambda: cached.cached_weigh(q, lse, c, b, out=w)), ("scaled_rows", lambda: scaled._launch("scaled_rows", (q,), None, None))):
        with pytest.raises(SparkError, match=name + " has no derivatives"):
            call()
    with torch.autograd.forward_ad.dual_level():
        dual = torch.autograd.forward_ad.make_dual(torch.ones(3), torch.ones(3))
        with pytest.raises(SparkError, match="cached_x has no derivatives"):
            scaled._launch("cached_x", (k, dual.as_subclass(On)), None, None)
    with pytest.raises(SparkError, match="8-bit rows has no derivatives"):
        scaled._no_gradient(q)
