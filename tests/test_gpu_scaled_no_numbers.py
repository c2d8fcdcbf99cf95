"""NaN and infinities in the rows and weights of products: they reach the outputs that they belong to, of either type and on every
way through the kernels, and no other."""
import pytest
import torch

from test_gpu_scaled import BF16, F32, activations, bits, ops, weights   # noqa: F401 (ops: the fixture)

pytestmark = pytest.mark.gpu

SIZES = [(1, 96, 640), (9, 40, 3584), (16, 60, 20000), (20, 48, 9000), (40, 96, 700), (77, 500, 1000), (130, 80, 384), (300, 700, 2500), (700, 300, 4100)]
NO_NUMBERS = (float("nan"), float("inf"), -float("inf"))


@pytest.mark.parametrize("m,n,k", SIZES)
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_products(ops, m, n, k, dtype):   # noqa: F811
    x, w = activations(m, k, m + k), weights(n, k, n + k, F32)
    rows, columns = ([0, m // 2, m - 1] if m > 4 else []), [1, n // 2, n - 1]
    clean_x, clean_w = x.clone(), w.clone()
    clean_x[rows] = 0.0
    clean_w[columns] = 0.0
    for i, v in enumerate(NO_NUMBERS):
        if rows:
            x[rows[i], (0, k // 2, k - 1)[i]] = v
        w[columns[i], (k - 1, 0, k // 3)[i]] = v
    got = ops.scaled_matmul(ops.scaled_rows(x.cuda()), ops.ScaledWeights(w.cuda()), dtype=dtype).cpu()
    clean = ops.scaled_matmul(ops.scaled_rows(clean_x.cuda()), ops.ScaledWeights(clean_w.cuda()), dtype=dtype).cpu()
    hit = torch.zeros(m, n, dtype=torch.bool)
    hit[rows] = True
    hit[:, columns] = True
    assert torch.equal(got.isnan(), hit)
    assert torch.equal(got[~hit], clean[~hit]) and bool(torch.isfinite(clean).all())


@pytest.mark.parametrize("m,n,k", [(1, 300, 640), (17, 130, 1500), (24, 200, 3584), (70, 300, 1000), (300, 200, 4100), (700, 130, 300)])
def test_pairs(ops, m, n, k):   # noqa: F811
    x, wg, wu = activations(m, k, m + k), weights(n, k, 1, F32), weights(n, k, 2, F32)
    clean = [wg.clone(), wu.clone()]
    wg[3, 5], wu[n // 2, k - 1], wg[n - 1, 0] = NO_NUMBERS
    columns = [3, n // 2, n - 1]
    for t in clean:
        t[columns] = 0.0
    rows = ops.scaled_rows(x.cuda())
    got = ops.scaled_gated(rows, ops.ScaledWeights(wg.cuda(), wu.cuda()))
    want = ops.scaled_gated(rows, ops.ScaledWeights(*(t.cuda() for t in clean)))
    nan = (bits(got.codes) & 127) == 127
    hit = torch.zeros_like(nan)
    hit[:, columns] = True
    assert torch.equal(nan, hit)
    assert torch.equal(bits(got.codes)[~hit], bits(want.codes)[~hit]) and torch.equal(bits(got.scales), bits(want.scales))
