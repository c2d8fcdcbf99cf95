"""What paper_2603_09215_amd/scaled.py refuses before it reaches the library or the GPU: on the CPU, with stand-ins for tensors that
no card could hold."""
import pytest
import torch

from paper_2603_09215_amd import SparkError, scaled


class Like:
    """a 2-d tensor on a GPU as far as the checks look; nothing lies behind it"""
    dtype, is_cuda, device, requires_grad = torch.bfloat16, True, torch.device("cuda", 0), False

    def __init__(self, m, k, **kw):
        self.shape = torch.Size((m, k))
        self.__dict__.update(kw)

    def stride(self):
        return self.shape[1], 1

    def data_ptr(self):
        return 1 << 20

    def get_device(self):
        raise AssertionError("reached the launch")


# the sizes' lower 32 bits would do
@pytest.mark.parametrize("m,k", [(1, (1 << 32) + 64), (1, (1 << 22) + 1), ((1 << 32) + 5, 64), (1 << 31, 64), ((1 << 64) // 128 + 3, 64)])
def test_sizes_past_32_bits(m, k):
    big = Like(m, k)
    for call in (lambda: scaled.scaled_rows(big), lambda: scaled.scaled_norm(big, torch.ones(4), 1e-6), lambda: scaled.ScaledRows.empty(m, k)):
        with pytest.raises(SparkError, match="are taken"):
            call()


def test_weights_past_32_bits():
    for n, k in (((1 << 32) + 16, 64), (16, (1 << 32) + 64), ((1 << 22) + 1, 64), (16, (1 << 22) + 1)):
        with pytest.raises(SparkError):
            scaled.ScaledWeights(Like(n, k))
        with pytest.raises(SparkError):
            scaled.ScaledWeights(Like(n, k), Like(n, k))


def test_a_products_rows_past_32_bits():
    w = object.__new__(scaled.ScaledWeights)
    w.n, w.k, w.pair, w._workspace = 16, 64, False, {}
    for m in ((1 << 32) + 8, 1 << 31, -1):
        with pytest.raises(SparkError, match="are taken"):
            w.workspace_bytes(m)


def test_rows_past_32_bits():
    codes, scales = torch.empty(0, 128, dtype=torch.float8_e4m3fn), torch.empty(0, 4, dtype=torch.float8_e8m0fnu)
    for k in ((1 << 32) + 64, 0, (1 << 22) + 1):
        with pytest.raises(SparkError, match="are taken"):
            scaled.ScaledRows(codes, scales, k)


def test_gradients_are_refused():
    """where torch keeps a graph (requires_grad) or tangents; under no_grad a parameter is a tensor as any other"""
    w = torch.nn.Parameter(torch.ones(4, 64))
    with pytest.raises(SparkError, match="no derivatives"):
        scaled._no_gradient(None, torch.ones(3), w)
    with torch.no_grad():
        scaled._no_gradient(w)
    scaled._no_gradient(w.detach(), None)
    with torch.autograd.forward_ad.dual_level():
        dual = torch.autograd.forward_ad.make_dual(torch.ones(4, 64), torch.ones(4, 64))
        with pytest.raises(SparkError, match="no derivatives"):
            scaled._no_gradient(dual)
        scaled._no_gradient(torch.ones(4, 64))
        with torch.no_grad(), pytest.raises(SparkError, match="no derivatives"):
            scaled._no_gradient(dual)


def test_every_launch_looks_for_gradients():
    """before anything is called, on the first tensor or another"""
    class On:
        requires_grad = False

        def get_device(self):
            return 0

    class Wanted(torch.Tensor):
        def get_device(self):
            return 0

    def never(*args):
        raise AssertionError("called")

    w = torch.ones(3).as_subclass(Wanted).requires_grad_()
    for tensors in ((w,), (On(), None, w)):
        with pytest.raises(SparkError, match="no derivatives"):
            scaled._launch("x", tensors, None, never)
