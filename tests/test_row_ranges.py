"""How the rows of a linear layer are shared out to launches where x or the residual reach 2 GiB (host code, compiled here)."""
import os
import random
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
DRIVER = r"""
#include <cstdio>
#include "tile_plan.hpp"
int main() {
  long m, k, n;
  while (std::scanf("%ld %ld %ld", &m, &k, &n) == 3) std::printf("%ld\n", tp::k::rows_a_launch(m, k, n));
}
"""


@pytest.fixture(scope="module")
def ranges(tmp_path_factory):
    cxx = shutil.which("g++")
    if not cxx:
        pytest.skip("no C++ compiler")
    d = tmp_path_factory.mktemp("rows")
    (d / "driver.cpp").write_text(DRIVER)
    subprocess.run([cxx, "-O1", "-std=c++17", "-I", os.path.join(ROOT, "paper_2306_03622_amd", "csrc", "kernels"),
                    str(d / "driver.cpp"), "-o", str(d / "driver")], check=True)
    return lambda shapes: [int(v) for v in subprocess.run([str(d / "driver")], input="\n".join("%d %d %d" % s for s in shapes),
                                                          check=True, capture_output=True, text=True).stdout.split()]


def test_every_range_is_below_2_gib(ranges):
    rng = random.Random(4)
    shapes = [(rng.randint(33, 2 ** rng.randint(6, 27)), 8 * rng.randint(1, 2 ** rng.randint(0, 11)), rng.choice((0, 64, 1024)))
              for _ in range(3000)]
    shapes += [(2 ** 31 // (2 * k) + d, k, 0) for k in (8, 64, 1000, 4096, 16384) for d in (-1, 0, 1)]      # around the limit
    for (m, k, n), rows in zip(shapes, ranges(shapes)):
        wide = 2 * max(k, n)
        assert 0 < rows <= m and rows * wide < 2 ** 31
        if m * wide < 2 ** 31:
            assert rows == m                        # one launch, as for any call below the limit
        else:
            assert rows % 256 == 0
            last = m - (-(-m // rows) - 1) * rows
            assert last > 32 and -(-m // rows) <= m * wide // (2 ** 31 - 256 * wide) + 1, (m, k, n, rows)


def test_rows_of_which_no_256_fit(ranges):
    assert ranges([(1000, 1 << 24, 0), (10, 1 << 24, 0), (64, 1 << 24, 0)]) == [0, 10, 0]
