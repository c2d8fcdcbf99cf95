"""How attention over a paged cache is cut (csrc/cached_plan.h, plain arithmetic): that a plan is one the launch has and fits its grid, and that the
sizes of tests/test_gpu_cached_long.py between them take every kernel, with one part and with several."""
import pathlib
import random
import subprocess

import pytest

from test_gpu_cached_long import LONG

CSRC = pathlib.Path(__file__).resolve().parent.parent / "paper_2603_09215_amd" / "csrc"
CUS = 256
DRIVER = r"""
#include <cstdio>
#include "cached_plan.h"
int main() {
  int fp32, hd, nkv, group, m, n, cus;
  long long slots;
  while (scanf("%d %d %d %d %d %d %lld %d", &fp32, &hd, &nkv, &group, &m, &n, &slots, &cus) == 8) {
    const spark::AttendPlan p = spark::attend_plan(fp32, hd, nkv, group, m, n, slots, cus);
    printf("%d %d %lld %d\n", p.pairs, p.splits, p.tiles, spark::MOST_SPLITS);
  }
}
"""


@pytest.fixture(scope="module")
def plans(tmp_path_factory):
    at = tmp_path_factory.mktemp("plan")
    (at / "plan.cpp").write_text(DRIVER)
    subprocess.run(["g++", "-O2", "-std=c++17", "-Wall", "-Werror", f"-I{CSRC}", "-o", str(at / "plan"), str(at / "plan.cpp")], check=True)

    def run(asked):   # (fp32, head_dim, kv heads, group, rows, sequences, slots, compute units)
        lines = "".join(" ".join(map(str, map(int, a))) + "\n" for a in asked)
        out = subprocess.run([str(at / "plan")], input=lines, capture_output=True, text=True, check=True).stdout
        return [tuple(map(int, line.split())) for line in out.splitlines()]
    return run


def test_plans_are_launches_that_there_are(plans):
    rng = random.Random(1)
    asked = []
    for _ in range(3000):
        nkv, group = rng.choice([1, 2, 4, 8, 40]), rng.choice([1, 2, 7, 16, 24, 100])
        n = int(2 ** rng.uniform(0, 14))
        m = min(int(2 ** rng.uniform(0, 22)), (1 << 26) // (nkv * group), 1 << 22)
        asked.append((rng.random() < 0.4, rng.choice([64, 128]), nkv, group, m, min(n, (1 << 20) // nkv), 16 * int(2 ** rng.uniform(0, 19)), rng.choice([256, 256, 304, 80])))
    asked.append((True, 128, 1, 1, 1 << 22, 1, 1 << 23, CUS))
    asked.append((True, 64, 16, 1, 1 << 22, 1 << 16, 1 << 23, CUS))
    for a, (pairs, splits, tiles, most) in zip(asked, plans(asked)):
        fp32, hd, nkv, group, m, n, slots, cus = a
        assert pairs == 16 or (not fp32 and pairs in (128, 2 * hd)), a
        assert 1 <= splits <= most
        assert (splits - 1) * (64 if pairs > 16 or fp32 else 128) < slots   # (every part has a step, where lengths fill the table)
        # room for any way in which m rows fall to n sequences
        full, rest = divmod(m, n)
        even = sum(-(-r * group // pairs) * c for r, c in ((full + 1, rest), (full, n - rest)))
        one = -(-max(1, m - n + 1) * group // pairs) + (-(-group // pairs)) * (min(n, m) - 1)
        assert tiles >= max(even, one), a
        assert tiles * nkv * splits * (512 if pairs == 256 else 256) < 1 << 32, a


def test_the_long_tests_take_every_kernel(plans):
    asked = [(dtype == "fp32", hd, nkv, nq // nkv, sum(r for r, _ in shape) + 3, len(shape), -(-max(c for _, c in shape) // page) * page, CUS)
             for shape, page, nq, nkv, hd, dtype, _ in LONG]
    seen = {(fp32, hd, pairs, splits > 1) for (fp32, hd, *_), (pairs, splits, _, _) in zip(asked, plans(asked))}
    for hd in (64, 128):
        for several in (False, True):
            assert (True, hd, 16, several) in seen
            for pairs in (16, 128, 256)[:hd // 64 + 1]:   # (heads of 64 have no tiles of 256)
                assert (False, hd, pairs, several) in seen, (hd, pairs, several)


def test_steps_of_32_dialogues_fill_the_card_and_prompts_take_tiles(plans):
    (pairs, splits, tiles, _), = plans([(False, 128, 2, 16, 32, 32, 8192, CUS)])
    assert pairs == 16 and tiles * 2 * splits >= CUS
    (pairs, splits, _, _), = plans([(False, 128, 4, 7, 8191, 1, 8192, CUS)])
    assert (pairs, splits) == (256, 1)
