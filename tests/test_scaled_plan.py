"""Which tiles products of 8-bit rows take (csrc/scaled_plan.h, plain arithmetic): that a plan is one the launch has, and that the
sizes of tests/test_gpu_scaled.py between them take every tile, over all of k and over parts of it."""
import pathlib
import random
import subprocess

import pytest

from test_gpu_scaled import GATED, MATMULS

CSRC = pathlib.Path(__file__).resolve().parent.parent / "paper_2603_09215_amd" / "csrc"
CUS = 256
DRIVER = r"""
#include <cstdio>
#include "scaled_plan.h"
int main() {
  int m, blocks, k, pair, fp32, cus;
  while (scanf("%d %d %d %d %d %d", &m, &blocks, &k, &pair, &fp32, &cus) == 6) {
    const spark::TilePlan p = spark::tile_plan(m, blocks, k, pair, fp32, cus);
    printf("%d %d %d %d\n", p.shape, p.splits, spark::TILE_SHAPES[p.shape].nt, spark::TILE_SHAPES[p.shape].mt);
  }
}
"""


@pytest.fixture(scope="module")
def plans(tmp_path_factory):
    at = tmp_path_factory.mktemp("plan")
    (at / "plan.cpp").write_text(DRIVER)
    subprocess.run(["g++", "-O2", "-std=c++17", "-Wall", "-Werror", f"-I{CSRC}", "-o", str(at / "plan"), str(at / "plan.cpp")], check=True)

    def run(asked):   # (m, n, k, pair, fp32, compute units)
        lines = "".join(f"{m} {-(-n // 16) * (1 + pair)} {k} {pair} {fp32} {cus}\n" for m, n, k, pair, fp32, cus in asked)
        out = subprocess.run([str(at / "plan")], input=lines, capture_output=True, text=True, check=True).stdout
        return [tuple(map(int, line.split())) for line in out.splitlines()]
    return run


def test_plans_are_launches_that_there_are(plans):
    rng = random.Random(1)

    def size(hi):
        return int(hi ** rng.random())
    asked = [(size(1 << 30), size(1 << 22), size(1 << 22), rng.randrange(2), 1, rng.choice((CUS, 304, 64, 1))) for _ in range(1000)]
    asked += [(m, n, k, 0, 0, cus) for m, n, k, _, _, cus in asked]
    for (m, n, k, pair, fp32, cus), (shape, splits, nt, mt) in zip(asked, plans(asked), strict=True):
        groups = -(-k // 512)
        assert shape in ((2, 3, 4, 5) if pair else (0, 1, 3, 4, 5))     # (gate and partner belong to one wave)
        assert 1 <= splits <= groups
        tiles = -(-(-(-n // 16) * (1 + pair)) // (8 * nt)) * -(-m // (16 * mt))
        assert splits == 1 or tiles * splits <= 2 * cus                   # so a launch's workgroups and its workspace are few


def test_sizes_of_the_gpu_tests_take_every_tile(plans):
    """(up to 16 rows a single matrix streams through registers, without a plan)"""
    singles = {(fp32, shape, splits > 1) for fp32 in (0, 1)
               for shape, splits, _, _ in plans([(m, n, k, 0, fp32, CUS) for m, n, k in MATMULS if m > 16])}
    assert singles == {(fp32, shape, cut) for fp32 in (0, 1) for shape in (0, 1, 3, 4, 5) for cut in (False, True)}
    pairs = {(shape, splits > 1) for shape, splits, _, _ in plans([(m, n, k, 1, 1, CUS) for m, n, k in GATED])}
    assert pairs == {(shape, cut) for shape in (2, 3, 4, 5) for cut in (False, True)}


def test_sizes_of_the_gpu_tests_take_the_stream_both_ways():
    """rows in LDS, up to 64 KiB of them, and rows that are read by each wave (scaled_stream_k)"""
    rows = {m * (-(-k // 128) * 128 + 16 + -(-(-(-k // 128)) // 4) * 4) <= 64 << 10 for m, n, k in MATMULS if m <= 16}
    assert rows == {False, True}
