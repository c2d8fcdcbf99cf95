"""Norms on their way into a paged cache with an eps past fp32's range (it is a 64-bit number)."""
import pytest
import torch

from test_gpu_cached_norms import normed

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("eps", [1e36, 3e38, 1e39, 1e60])
def test_large_eps(eps):
    normed(1.0, eps ** 0.5 if eps < 1e50 else 1e30, eps, torch.float32)
    normed(1e10, 1e20, eps, torch.bfloat16, hd=128)


def test_small_eps():
    normed(1e-20, 1.0, 1e-50, torch.float32)
    normed(0.0, 1.0, 1e-50, torch.float32)
