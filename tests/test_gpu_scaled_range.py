"""The operators on 8-bit rows at the ends of fp32's range: what is finite there comes back finite, with its bits.

Outputs in fp32 are the 64-bit sums, off by (blocks + 17) 2^-22 of their magnitudes and half a step as everywhere
(tests/test_gpu_scaled.py), and by 2^-118 of the largest power of their row of weights for every block and part (a sum is held
in steps of 2^-150 there, 2^-32 and that power below the outputs), and by half of fp32's smallest number."""
import pytest
import torch

import scaled_ref as ref
from test_gpu_scaled import activations, bits, check_gated, held, ops, product_bound   # noqa: F401 (ops: the fixture)
from test_gpu_scaled import F32

pytestmark = pytest.mark.gpu

SHAPES = [(1, 96, 640), (9, 40, 3584), (12, 33, 21800), (40, 96, 640), (20, 48, 9000), (130, 80, 384), (300, 200, 1000), (700, 300, 4100)]


def drawn(m, k, seed, size, same_sign=False):
    v = torch.randn(m, k, generator=torch.Generator().manual_seed(seed), dtype=torch.float64)
    v = v.clamp(-4, 4)
    return ((v.abs() + 0.5 if same_sign else v) * size).float()


def check(ops, x, w):   # noqa: F811
    m, k = x.shape
    want, mags = ref.product(held(x), held(w))
    assert bool((mags < 3.4e38).all())
    out = ops.scaled_matmul(ops.scaled_rows(x.cuda()), ops.ScaledWeights(w.cuda())).cpu().double()
    blocks = ref.padded(k)[0]
    err, half = product_bound(blocks, mags, F32)
    top = 2.0 ** (ref.quantise(w.double())[1][:, :blocks].amax(1).double() - 127)
    err = err + (blocks + 17) * 2.0 ** -118 * top + 2.0 ** -150
    assert bool(torch.isfinite(out).all()), int((~torch.isfinite(out)).sum())
    assert bool(((out - want).abs() <= err + half * (want.abs() + err)).all()), float(((out - want).abs() / mags).max())


@pytest.mark.parametrize("m,n,k", SHAPES)
@pytest.mark.parametrize("xs,ws", [(1e-20, 1e-16), (1e-22, 1e-15), (1.0, 1e-36), (1e-5, 1e-31), (1e-28, 1e-9), (1e-30, 1e-3), (1e-25, 1e25), (1e-30, 1e33)])
def test_small_rows_and_small_outputs(ops, m, n, k, xs, ws):   # noqa: F811
    check(ops, drawn(m, k, 1, xs), drawn(n, k, 2, ws))


@pytest.mark.parametrize("m,n,k", SHAPES)
@pytest.mark.parametrize("xs,ws", [(6e37, 1e-8), (6e37, 1e-5), (6e37, 1e-38), (1e30, 1e3), (1e-3, 1e36), (1.0, 2e33)])
def test_large_rows_of_one_sign(ops, m, n, k, xs, ws):   # noqa: F811
    check(ops, drawn(m, k, 1, xs, True), drawn(n, k, 2, ws, True))


@pytest.mark.parametrize("m,n,k", SHAPES)
@pytest.mark.parametrize("size", [1e-38, 1e-20, 1e-8, 1e-5])
def test_rows_of_the_largest_numbers(ops, m, n, k, size):   # noqa: F811
    g = torch.Generator().manual_seed(1)
    check(ops, 3.3e38 * (1 + 0.03 * torch.rand(m, k, generator=g)), size * (1 + 0.03 * torch.rand(n, k, generator=g)))


@pytest.mark.parametrize("m", [1, 20])
def test_the_longest_row_of_the_largest_numbers(ops, m):   # noqa: F811
    """all of fp32's largest, 2^22 of them, one sign: every partial sum is finite because the whole is"""
    k = 1 << 22
    x, w = torch.full((m, k), 3.4e38), torch.full((3, k), 1e-10)
    out = ops.scaled_matmul(ops.scaled_rows(x.cuda()), ops.ScaledWeights(w.cuda())).cpu().double()
    want = held(x[:1, :128])[0, 0] * held(w[:1, :128])[0, 0] * k
    assert bool(((out / want - 1).abs() <= (k // 128 + 17) * 2.0 ** -22).all()), out


@pytest.mark.parametrize("m,n,k", [(1, 200, 640), (24, 200, 3584), (70, 300, 1000), (300, 200, 4100)])
@pytest.mark.parametrize("xs,gs,us", [(1e-20, 1e18, 1e-13), (6e37, 1e-36, 1e-9), (1e-28, 1e27, 1e20), (1e30, 1e-32, 1e2)])
def test_gated_of_small_and_large_rows(ops, m, n, k, xs, gs, us):   # noqa: F811
    """sums near 1 of the gate, sums of the other at the ends of the range"""
    x, wg, wu = drawn(m, k, 1, xs, True), drawn(n, k, 2, gs / k ** 0.5), drawn(n, k, 3, us, True)
    rows = ops.scaled_gated(ops.scaled_rows(x.cuda()), ops.ScaledWeights(wg.cuda(), wu.cuda()))
    assert not bool(((bits(rows.codes) & 127) == 127).any())
    check_gated(rows, x, wg, wu, n, k)
