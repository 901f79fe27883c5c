"""How tps_lora takes its rows where scratch does not hold all of their inner sums (host code, compiled here), and what the header says of it."""
import os
import random
import re
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
DRIVER = r"""
#include <cstdio>
#include "lora_plan.hpp"
using namespace tp::k;
int main() {
  long m, n, k, r, adapters;
  unsigned long scratch;
  while (std::scanf("%ld %ld %ld %ld %ld %lu", &m, &n, &k, &r, &adapters, &scratch) == 6) {
    const long rows = lora_rows(m, n, k, r, adapters, scratch);
    const LoraPlan p = lora_plan(rows < m ? rows : m, n, k, r, adapters, scratch);
    std::printf("%ld %d %d\n", rows, p.splits, p.order);
  }
}
"""
SCRATCH = 32 << 20


@pytest.fixture(scope="module")
def parts(tmp_path_factory):
    cxx = shutil.which("g++")
    if not cxx:
        pytest.skip("no C++ compiler")
    d = tmp_path_factory.mktemp("lora_parts")
    (d / "driver.cpp").write_text(DRIVER)
    subprocess.run([cxx, "-O1", "-std=c++17", "-I", os.path.join(ROOT, "paper_2306_03622_amd", "csrc", "kernels"),
                    str(d / "driver.cpp"), "-o", str(d / "driver")], check=True)

    def run(calls):
        out = subprocess.run([str(d / "driver")], input="\n".join(" ".join(str(int(v)) for v in c) for c in calls), check=True,
                             capture_output=True, text=True).stdout
        return [tuple(int(v) for v in line.split()) for line in out.splitlines()]

    return run


def test_the_border_of_the_usual_scratch(parts):
    # (rows, rank): the last that 32 MiB hold at once, and the first that they do not
    calls = [(m, 4096, 4096, r, 32, SCRATCH) for m, r in ((64527, 128), (64528, 128), (65536, 128), (65537, 128), (127100, 64), (127101, 64), (200000, 64))]
    got = parts(calls)
    assert [g[0] for g in got] == [64527, 32320, 32768, 32832, 127100, 63552, 100032]
    assert all(splits >= 1 and order == 1 for _, splits, order in got)       # two launches, rows in order
    # no more adapters than are found in a tile: nothing but the inner sums has to fit
    assert parts([(65536, 4096, 4096, 128, 1, SCRATCH), (65537, 4096, 4096, 128, 1, SCRATCH)]) == [(65536, 1, 0), (32832, 1, 0)]


def test_little_scratch(parts):
    size = lambda rows, r: 4 * rows * (r + 2)                                   # noqa: E731
    # parts of 1024 rows (4096 where one launch computes the inner sums once), else one launch
    assert parts([(5000, 1024, 1024, 64, 3, size(1024, 64)), (5000, 1024, 1024, 64, 3, size(1024, 64) - 4),
                  (9000, 256, 1024, 64, 3, size(4608, 64)), (9000, 256, 1024, 64, 3, size(4000, 64)), (5000, 1024, 1024, 64, 3, 0)]) == \
        [(1024, 1, 2), (5000, 0, 0), (4544, 1, 2), (9000, 0, 0), (5000, 0, 0)]


def test_parts_hold_all_rows(parts):
    rng = random.Random(14)
    calls = [(2 ** rng.randint(0, 30) + rng.randint(0, 99), 2 ** rng.randint(0, 13), 8 * 2 ** rng.randint(0, 10), 8 * rng.randint(1, 16),
              rng.choice((1, 2, 5, 8, 100, 5000)), rng.choice((0, 4096, 2 ** rng.randint(10, 30), SCRATCH, 2 ** 40))) for _ in range(20000)]
    for c, (rows, splits, order) in zip(calls, parts(calls)):
        m, n, _, r, _, scratch = c
        if (m + 15) // 16 * ((n + 255) // 256) >= 1 << 24:
            continue                                             # refused before
        assert 1 <= rows <= m, c
        if rows < m:
            assert rows % 64 == 0 and rows >= 1024 and splits >= 1 and 4 * rows * (splits * r + (2 if order else 0)) <= scratch, c
            assert -(-m // rows) == -(-m // (min(scratch // (4 * (r + 2)), 2 ** 27 - 1) // 64 * 64)), c       # no more than have to be
        elif m >= 4096 and scratch >= 4 * 4160 * (r + 2):
            assert splits >= 1, c


def test_the_header_promises_no_more():
    src = open(os.path.join(ROOT, "include", "torpor_serve.h")).read()
    assert not re.search(r"TPO_WORK_BYTES\s+is as much as any call uses", src)
