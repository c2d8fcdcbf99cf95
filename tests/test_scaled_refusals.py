"""The operators on 8-bit rows without a GPU: sizes in closed form, and arguments that are refused before anything is
launched (the pointers are made up: nothing reads them)."""
import ctypes as C

import pytest

from paper_2603_09215_amd import binding as sb

EINVAL, ENOMEM = -1, -3
P = 1 << 20   # an aligned address that nothing follows


@pytest.fixture(scope="module")
def lib():
    return sb.load_library()


@pytest.mark.parametrize("n,k", [(1, 1), (16, 128), (17, 129), (4608, 3584), (1001, 1000), (1 << 22, 1)])
def test_weight_bytes(lib, n, k):
    for pair in (0, 1):
        blocks = -(-k // 128)
        rows = -(-n // 16) * (1 + pair)
        size = C.c_size_t()
        assert lib.spark_scaled_weight_bytes(n, k, pair, C.byref(size)) == 0
        assert size.value == rows * (blocks * 2048 + -(-blocks // 4) * 4 * 16 + 16)


def test_sizes_are_refused(lib):
    size = C.c_size_t()
    for n, k in ((0, 5), (5, 0), (-1, 5), ((1 << 22) + 1, 5), (5, (1 << 22) + 1)):
        assert lib.spark_scaled_weight_bytes(n, k, 0, C.byref(size)) == EINVAL
        assert lib.spark_scaled_workspace_bytes(1, n, k, 0, C.byref(size)) == EINVAL
        assert lib.spark_scaled_pack(P, None, 1, 1 << 25, n, k, P, 1 << 40, None) == EINVAL
        assert lib.spark_scaled_matmul(P, P, 1, P, n, k, P, 0, 1 << 25, None, 0, None) == EINVAL
        assert lib.spark_scaled_gated(P, P, 1, P, n, k, P, P, None, 0, None) == EINVAL
    assert lib.spark_scaled_weight_bytes(4, 4, 0, None) == EINVAL
    assert lib.spark_scaled_workspace_bytes(-1, 4, 4, 0, C.byref(size)) == EINVAL
    assert lib.spark_scaled_workspace_bytes(1, 4, 4, 0, None) == EINVAL
    for k in (0, -3, (1 << 22) + 1):
        assert lib.spark_scaled_rows(P, 0, 1 << 25, 1, k, P, P, None) == EINVAL
        assert lib.spark_scaled_norm(P, 0, 1 << 25, None, 0, 0, P, 1 << 25, P, 1e-6, 1, k, P, P, None) == EINVAL


def test_rows_arguments(lib):
    good = [P, 0, 64, 3, 64, P, P, None]
    for at, bad in ((0, None), (0, P + 2), (1, 2), (1, -1), (2, 63), (2, -64), (3, -1), (5, None), (5, P + 8), (6, None), (6, P + 2)):
        args = list(good)
        args[at] = bad
        assert lib.spark_scaled_rows(*args) == EINVAL, (at, bad)
    assert lib.spark_scaled_rows(P, 0, 64, 0, 64, P, P, None) == 0   # no rows: nothing to launch


def test_norm_arguments(lib):
    good = [P, 0, 64, P, 1, 64, P, 64, P, 1e-6, 3, 64, P, P, None]
    for at, bad in ((0, None), (0, P + 1), (1, 5), (2, 10), (3, P + 1), (4, 7), (5, 63), (6, None), (7, 63), (7, 80), (8, None), (8, P + 2), (9, -1.0),
                    (9, float("nan")), (10, -1), (12, None), (12, P + 4), (13, None), (13, P + 1)):
        args = list(good)
        args[at] = bad
        assert lib.spark_scaled_norm(*args) == EINVAL, (at, bad)
    args = list(good)
    args[10] = 0
    assert lib.spark_scaled_norm(*args) == 0
    args[3:6] = None, 99, -5   # without y its type and stride say nothing
    assert lib.spark_scaled_norm(*args) == 0


def test_pack_arguments(lib):
    size = C.c_size_t()
    assert lib.spark_scaled_weight_bytes(20, 64, 0, C.byref(size)) == 0
    good = [P, None, 1, 64, 20, 64, P, size.value, None]
    for at, bad, code in ((0, None, EINVAL), (0, P + 1, EINVAL), (1, P + 1, EINVAL), (2, 3, EINVAL), (3, 63, EINVAL), (6, None, EINVAL),
                          (6, P + 8, EINVAL), (7, size.value - 1, ENOMEM)):
        args = list(good)
        args[at] = bad
        assert lib.spark_scaled_pack(*args) == code, (at, bad)
    args = list(good)
    args[1] = P   # a pair needs twice the room
    assert lib.spark_scaled_pack(*args) == ENOMEM


def test_product_arguments(lib):
    good = [P, P, 3, P, 20, 64, P, 0, 20, None, 0, None]
    for at, bad in ((0, None), (0, P + 8), (1, None), (1, P + 2), (2, -1), (3, None), (3, P + 8), (6, None), (6, P + 2), (7, 2), (8, 19)):
        args = list(good)
        args[at] = bad
        assert lib.spark_scaled_matmul(*args) == EINVAL, (at, bad)
    good = [P, P, 3, P, 20, 64, P, P, None, 0, None]
    for at, bad in ((0, None), (0, P + 8), (1, None), (1, P + 2), (2, -1), (3, None), (3, P + 8), (6, None), (6, P + 8), (7, None), (7, P + 2)):
        args = list(good)
        args[at] = bad
        assert lib.spark_scaled_gated(*args) == EINVAL, (at, bad)


def test_model_bytes(lib):
    import workloads as wl
    w = wl.STEP_AUDIO_2_MINI
    size = C.c_size_t()
    cfg = sb.make_config(w.shape, w.schedule, 1, 2048, 64)
    assert lib.spark_scaled_model_bytes(C.byref(cfg), C.byref(size)) == 0
    weights = 28 * (4608 * 3584 + 3584 * 3584 + 3 * 18944 * 3584)   # a byte each, and powers, rows and parts
    assert weights < size.value < 1.02 * weights + (128 << 20)
    assert lib.spark_scaled_model_bytes(C.byref(cfg), None) == EINVAL
    cfg = sb.make_config(wl.TINY.shape, wl.TINY.schedule, 1, 64, 16)   # fp32
    assert lib.spark_scaled_model_bytes(C.byref(cfg), C.byref(size)) == EINVAL
    assert lib.spark_scaled_projections(None, P, 1 << 40) == EINVAL
