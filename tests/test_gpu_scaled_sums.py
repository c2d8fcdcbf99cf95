"""The residual's sum that the norm stores, element by element, and products as a whole: relative 2-norms beside the bounds of
single elements, and inputs on which nothing is lost, where outputs are the 64-bit ones rounded once.  The checks are those
of tests/scaled_checks.py."""
import pytest
import torch

import scaled_checks as ck
import scaled_ref as ref
from scaled_checks import BF16, F32
from test_gpu_scaled import MATMULS, activations, held, ops, same_rows, weights   # noqa: F401 (ops: the fixture)

pytestmark = pytest.mark.gpu


def sums(ops, h, y, gain, eps, in_place):   # noqa: F811
    """rows and stored sums of one call, both against 64 bits"""
    want = ck.residual_sum(h, y)
    dev = h.cuda()
    out = dev if in_place else torch.full_like(dev, -7.0)
    rows = ops.scaled_norm(dev, gain.cuda(), eps, y=None if y is None else y.cuda(), h_out=None if in_place else out)
    assert ck.same_values(out.cpu(), want)
    assert in_place or ck.same_values(dev.cpu(), h)
    v = want / torch.sqrt((want * want).mean(1, keepdim=True) + eps) * gain.double()
    same_rows(rows, *ref.quantise(v))


@pytest.mark.parametrize("m,k", [(1, 1), (3, 130), (5, 2500), (1, 3584), (9, 4096), (4, 4104), (2, 9000), (2, 18944), (3, 20001), (300, 256)])
@pytest.mark.parametrize("dtype,ytype", [(F32, F32), (F32, BF16), (BF16, BF16), (BF16, F32), (F32, None), (BF16, None)])
@pytest.mark.parametrize("in_place", [True, False])
def test_stored_sums(ops, m, k, dtype, ytype, in_place):   # noqa: F811
    h = activations(m, k, m + k, dtype)
    y = None if ytype is None else activations(m, k, m + k + 1, ytype, 1.0)
    sums(ops, h, y, 1 + 0.1 * torch.randn(k, generator=torch.Generator().manual_seed(k)), 1e-6, in_place)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("ytype", [F32, BF16])
def test_stored_sums_beside_the_middles(ops, dtype, ytype):   # noqa: F811
    """h + y at the middle between two bf16 numbers and a little beside it, further down than an fp32 sum can hold; cancelling;
    below the smallest normal number"""
    h = torch.tensor([256.0, 258.0, 1.0, -3.0, 2.0 ** -126, 1e30, 2.0 ** -130]).repeat_interleave(64)
    unit = 2.0 ** (torch.frexp(h.abs())[1].float().clamp(min=-125) - 9)
    off = torch.cat([torch.tensor([0.0, 1.0, -1.0]), 2.0 ** -torch.arange(7.0, 35.0), -2.0 ** -torch.arange(7.0, 35.0), torch.zeros(5)]).repeat(7)
    y = torch.stack([unit * (1 + off), -unit * (1 + off), unit * 0.5 * (1 + off), unit * off, h * off, -h]).to(ytype)
    sums(ops, h.expand(6, -1).contiguous().to(dtype), y, torch.ones(448), 1e-6, False)


@pytest.mark.parametrize("dtype,ytype", [(F32, F32), (BF16, F32), (BF16, BF16)])
def test_stored_sums_of_special_values(ops, dtype, ytype):   # noqa: F811
    inf, nan = float("inf"), float("nan")
    pairs = torch.tensor([(0.0, -0.0), (inf, 1.0), (inf, -inf), (nan, 1.0), (1.0, nan), (3e38, 3e38), (-3e38, -3e38), (3e38, -3e38), (1e-40, 1e-40), (5.0, 1e-30)])
    h, y = (pairs[:, i, None].repeat(1, 136).to(t) for i, t in ((0, dtype), (1, ytype)))
    sums(ops, h, y, torch.ones(136), 1e-6, True)


@pytest.mark.parametrize("m,n,k", [s for s in MATMULS if s[0] * s[1] >= 400])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_products_as_a_whole(ops, m, n, k, dtype):   # noqa: F811
    x, w = activations(m, k, m + 3 * n + k), weights(n, k, n + k)
    out = ops.scaled_matmul(ops.scaled_rows(x.cuda()), ops.ScaledWeights(w.cuda()), dtype=dtype).cpu()
    off = ck.beyond_rounding(out, ref.product(held(x), held(w))[0], dtype)
    print(f"  {m} x {n} x {k} {dtype}: {off:.2e} beyond rounding, {ck.sum_tolerance(k, dtype):.2e} allowed", flush=True)
    assert off <= ck.sum_tolerance(k, dtype)


EXACT = [(1, 100, 129), (7, 257, 3584), (16, 96, 16384), (12, 40, 21800), (17, 129, 1100), (33, 500, 2048), (77, 1001, 1000), (130, 300, 4096), (300, 700, 2500), (1023, 520, 4100)]


@pytest.mark.parametrize("m,n,k", EXACT)
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_products_where_nothing_is_lost(ops, m, n, k, dtype):   # noqa: F811
    x, w = ck.one_binade(m, k, 1, torch.arange(m)[:, None] % 9 - 4), ck.one_binade(n, k, 2, torch.arange(n)[:, None] % 5 - 9)
    out = ops.scaled_matmul(ops.scaled_rows(x.cuda()), ops.ScaledWeights(w.cuda()), dtype=dtype).cpu()
    want = ref.to_type(ref.product(x.double(), w.double())[0], dtype)
    assert ck.same_values(out, want)
