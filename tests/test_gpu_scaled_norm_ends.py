"""The norm into 8-bit rows where a row is no numbers, and where its values pass fp32's range."""
import pytest
import torch

from test_gpu_scaled import BF16, F32, activations, bits, norm_case, ops   # noqa: F401 (ops: the fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("k", [1, 7, 136, 300, 3000, 9000, 20001])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_zeros_behind_rows_that_are_no_numbers(ops, k, dtype):   # noqa: F811
    h = activations(5, k, k, dtype)
    h[1, k // 2] = float("nan")
    h[2, 0] = float("inf")
    h[3] = 0.0                       # 0 / 0 with eps 0
    rows = ops.scaled_norm(h.cuda(), torch.ones(k, device="cuda"), 0.0)
    assert not bool(bits(rows.codes)[:, k:].any())
    assert bool(((bits(rows.codes)[1:4:2, :k] & 127) == 127).all())
    norm_case(ops, h, None, torch.ones(k), 0.0)


@pytest.mark.parametrize("k", [64, 512, 3584, 4096, 9000, 1 << 20])
def test_norms_beyond_fp32(ops, k):   # noqa: F811
    """gains that take the norm past fp32's largest number: 8-bit rows hold up to 448 * 2^127, and what is beyond that is that"""
    g = torch.Generator().manual_seed(k)
    h = torch.randn(4, k, generator=g)
    h[1] = 0.0
    h[1, k // 2] = 1.0                 # the norm is sqrt(k) there
    h[2, ::3] *= 1e-30
    gain = torch.randn(k, generator=g).clamp(-3, 3) * 1e38
    gain[1::5] = 1e-3
    gain[2::7] = 3.4e38
    gain[k // 2] = -3.4e38
    norm_case(ops, h, None, gain, 0.0)
    gain[3] = float("inf")
    norm_case(ops, h, None, gain, 1e-6)
    norm_case(ops, h.bfloat16(), None, gain, 1e-6)
