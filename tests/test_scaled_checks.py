"""The checks of tests/scaled_checks.py on the CPU: what is right passes, and each planted mistake is caught."""
import pytest
import torch

import scaled_checks as ck
import scaled_ref as ref
from scaled_checks import BF16, F32


def inputs(m, n, k):
    g = torch.Generator().manual_seed(m + n + k)
    x = torch.randn(m, k, generator=g) * torch.exp(torch.randn(m, 1, generator=g))
    x[:, torch.rand(k, generator=g) < 0.01] *= 30
    w = torch.randn(n, k, generator=g) * 0.02
    return (ref.values(*ref.quantise(v.double())) for v in (x, w))


@pytest.mark.parametrize("dtype,ytype", [(F32, F32), (F32, BF16), (BF16, BF16), (BF16, F32)])
def test_residual_sums(dtype, ytype):
    g = torch.Generator().manual_seed(1)
    h, y = torch.randn(5, 300, generator=g).to(dtype), torch.randn(5, 300, generator=g).to(ytype)
    h[0, 3] = float("nan")
    want = ck.residual_sum(h, y)
    got = (h.double() + y.double()).to(dtype)
    if dtype == F32:
        assert ck.same_values(got, want)
    wrong = want.to(dtype)
    assert ck.same_values(wrong, want)
    bits = wrong.view(torch.int32 if dtype == F32 else torch.int16)
    bits[4, 299] += 1                                     # one element off by its last bit
    assert not ck.same_values(wrong, want)
    assert not ck.same_values(torch.where(want.isnan(), 0.0, want), want)
    assert not ck.same_values(h, want)                    # never added
    assert ck.residual_sum(torch.full((1, 1), 3.3e38, dtype=dtype), torch.full((1, 1), 1e38, dtype=ytype)).isinf().all()


@pytest.mark.parametrize("m,n,k", [(12, 100, 21800), (16, 200, 16384), (65, 16, 4096), (8, 257, 513)])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_products(m, n, k, dtype):
    x, w = inputs(m, n, k)
    want, allowed = ref.product(x, w)[0], ck.sum_tolerance(k, dtype)
    right = ref.to_type(want, dtype)
    assert ck.beyond_rounding(right, want, dtype) == 0.0
    lost = x.clone()
    lost[:, k - 8:] = 0.0
    down = torch.where(right.abs() > want.abs(), 1.0, 0.0)   # cut toward zero and not rounded
    cut = right - torch.copysign(down * 2.0 ** (torch.frexp(want)[1].double() - (24 if dtype == F32 else 8)), want)
    wrongs = {"the last eight of k": ref.to_type(ref.product(lost, w)[0], dtype), "1 %": ref.to_type(want * 1.01, dtype),
              "not a number": torch.where(torch.arange(n) == 3, float("nan"), right)}
    if dtype == BF16:
        wrongs["cut, not rounded"] = cut
    for what, got in wrongs.items():
        assert ck.beyond_rounding(got, want, dtype) > 2 * allowed, what


def test_one_binade_loses_nothing():
    for k in (100, 5000):
        x, w = ck.one_binade(9, k, 1, torch.arange(-4, 5)[:, None]), ck.one_binade(33, k, 2)
        for v in (x, w):
            assert torch.equal(ref.values(*ref.quantise(v.double()))[:, :k], v.double())
        want = ref.product(x.double(), w.double())[0]
        assert torch.equal(want, want.float().double())
        # neighbours' products lie in one binade and a bit: their last bit is not 13 below the largest's first
        p = (x[0].double() * w[0].double()).abs()
        assert float(p.max() / p.min()) < 4 and torch.equal(p * 2.0 ** 10, torch.round(p * 2.0 ** 10))
