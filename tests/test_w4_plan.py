"""The plan of the 4-bit linear layers (host code, compiled here): every call within the documented sizes takes a kernel whose grid
can be launched, and larger ones are refused."""
import ctypes
import os
import shutil
import subprocess

import pytest

import paper_2306_03622_amd as tp
from tests.test_ops_host import linear_args

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
DRIVER = r"""
#include <cstdio>
#include "w4_plan.hpp"
using namespace tp::k;
int main() {
  long m, n, k;
  int g;
  for (int i = 0; i < W4_VARIANTS; ++i) std::printf("%d %d %d\n", kW4[i].bn, kW4[i].bm, kW4[i].threads);
  while (std::scanf("%ld %ld %ld %d", &m, &n, &k, &g) == 4) std::printf("%d\n", w4_plan(m, n, k, g));
}
"""
ROWS = 3                                 # the first variants: row tiles in a grid's second dimension


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    cxx = shutil.which("g++")
    if not cxx:
        pytest.skip("no C++ compiler")
    d = tmp_path_factory.mktemp("w4_plan")
    (d / "driver.cpp").write_text(DRIVER)
    subprocess.run([cxx, "-O1", "-std=c++17", "-I", os.path.join(ROOT, "paper_2306_03622_amd", "csrc", "kernels"),
                    str(d / "driver.cpp"), "-o", str(d / "driver")], check=True)

    def run(shapes):                     # (M, N, K, group) -> variants' (outputs, rows, threads), plans
        out = subprocess.run([str(d / "driver")], input="\n".join(" ".join(map(str, s)) for s in shapes), check=True,
                             capture_output=True, text=True).stdout.splitlines()
        split = len(out) - len(shapes)
        return [tuple(map(int, v.split())) for v in out[:split]], [int(v) for v in out[split:]]

    return run


def up(a, b):
    return -(-a // b)


def test_every_plan_can_be_launched(plan):
    shapes = [(m, n, k, g) for m in (1, 16, 1000, 65536, 1048560, 1048561, 1100000, 1500000, 2 * 10 ** 6, 3 * 10 ** 6, 10 ** 7, 10 ** 8,
                                     2 ** 29, 2 ** 30 - 128)
              for n in (1, 7, 16, 17, 32, 33, 64, 128, 1000, 4096, 50000, 2 ** 24) for g in (32, 64, 128)
              for k in (*range(g, 2049, g), 4096, 2 ** 20) if up(m, 128) * up(n, 256) < 2 ** 23]
    variants, plans = plan(shapes)
    for (m, n, k, g), p in zip(shapes, plans):
        assert 0 <= p < len(variants), (m, n, k, g)
        bn, bm, threads = variants[p]
        if p < ROWS:
            assert up(m, bm) <= 65535 and up(n, bn) * threads < 2 ** 32, (m, n, k, g, p)
        else:
            assert up(m, bm) * up(n, bn) * threads < 2 ** 32, (m, n, k, g, p)


def test_the_gpu_shapes_reach_every_kernel_with_every_group(plan):
    from tests.test_gpu_linear_w4 import SHAPES
    from tests.test_gpu_linear_w4_variants import SHAPES as MORE
    shapes = [*SHAPES, *MORE]
    variants, plans = plan(shapes)
    assert {(p, s[3]) for s, p in zip(shapes, plans)} == {(p, g) for p in range(len(variants)) for g in (32, 64, 128)}


@pytest.mark.parametrize("m,n", [(2 ** 30 - 127, 1), (2 ** 31 - 1, 1), (2 ** 31 - 1, 2 ** 24), (2 ** 14, 2 ** 24), (2 ** 29, 257)])
def test_more_outputs_are_refused(m, n):
    a = linear_args(M=m, N=n, ldy=n)     # (addresses that are never read: refused before a launch)
    L = tp.lib()
    assert L.tpo_linear_w4(ctypes.byref(a), None) == tp.TP_E_INVAL
    assert "2^38" in L.tp_last_error().decode()
