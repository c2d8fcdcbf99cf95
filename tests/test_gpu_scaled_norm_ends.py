"""The norm into 8-bit rows where a row is no numbers, and where its values pass fp32's range."""
import pytest
import torch

import scaled_ref as ref
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
