"""The plan of rows in and out of a paged cache (host code, compiled here): the GPU tests' shapes reach every kernel and column split, and
every call within the documented sizes gets a grid that can be launched and that covers its rows once."""
import os
import random
import shutil
import subprocess

import pytest

from tests.test_gpu_cache_rows_variants import ROWS

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
DRIVER = r"""
#include <cstdio>
#include "cache_plan.hpp"
int main() {
  long dim, heads, batch, rows;
  while (std::scanf("%ld %ld %ld %ld", &dim, &heads, &batch, &rows) == 4) {
    const auto p = tp::k::cache_rows_plan((int)dim, heads, batch, rows);
    std::printf("%d %d %d %d %ld\n", p.per, p.cols, p.rows, p.each, (long)p.blocks);
  }
}
"""


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    cxx = shutil.which("g++")
    if not cxx:
        pytest.skip("no C++ compiler")
    d = tmp_path_factory.mktemp("cache_rows_plan")
    (d / "driver.cpp").write_text(DRIVER)
    subprocess.run([cxx, "-O1", "-std=c++17", "-I", os.path.join(ROOT, "paper_2306_03622_amd", "csrc", "kernels"),
                    str(d / "driver.cpp"), "-o", str(d / "driver")], check=True)

    def run(calls):
        out = subprocess.run([str(d / "driver")], input="\n".join(" ".join(str(v) for v in c) for c in calls), check=True,
                             capture_output=True, text=True).stdout
        return [tuple(int(v) for v in line.split()) for line in out.splitlines()]

    return run


def test_the_gpu_shapes_reach_every_kernel(plan):
    reached = set()
    for shape, (_, cols, rows, each, _) in zip(ROWS, plan([(dim, heads, len(lens), q_len) for _, dim, heads, _, q_len, lens, _ in ROWS])):
        assert (each, cols, rows) == shape[0], (shape, each, cols, rows)
        reached.add((shape[1], each, min(cols, 2)))
    assert reached == {(dim, each, cols) for dim in (64, 128) for each in (1, 2) for cols in (1, 2)}


def test_rows_are_covered_once(plan):
    rng = random.Random(15)
    calls = [(64, 1, (1 << 22) - 1, 15), (128, 65535, 1, 1023), (128, 9, 1, ((1 << 26) - 1) // 9), (64, 33, 1, ((1 << 26) - 1) // 33)]
    while len(calls) < 20000:
        heads, batch, rows = 2 ** rng.randint(0, 15) + rng.randint(0, 3), 2 ** rng.randint(0, 20) + rng.randint(0, 3), 2 ** rng.randint(0, 20) + rng.randint(0, 3)
        if batch * rows * heads < 1 << 26 and batch * heads < 1 << 22:           # others are refused before
            calls.append((rng.choice((64, 128)), heads, batch, rows))
    for (dim, heads, batch, q_len), (per, cols, rows, each, blocks) in zip(calls, plan(calls)):
        assert per == heads * dim // 8 and cols == -(-per // 256) and (rows == 1 if cols > 1 else 1 <= rows == 256 // per)
        assert each in (1, 2) and blocks == -(-q_len // (rows * each))
        assert blocks * cols * batch < 1 << 24
