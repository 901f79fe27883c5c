"""The plan of the masked attention (host code, compiled here): the GPU tests' shapes reach every kernel, with split keys and without,
and every call within the documented sizes gets a grid that can be launched and splits that its scratch holds."""
import os
import random
import shutil
import subprocess

import pytest

from tests.test_gpu_attention_variants import SHAPES

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
KERNELS = ["ATTN64_R32", "ATTN64_R64", "ATTN64_R128", "ATTN64_R128_LONG", "ATTN128_R32", "ATTN128_R64", "ATTN128_R128_DEEP",
           "ATTN128_R128", "ATTN128_R256"]
ROWS = [32, 64, 128, 128, 32, 64, 128, 128, 256]                 # of a workgroup
THREADS = [256, 256, 256, 256, 256, 256, 512, 256, 512]
SPLIT = {"ATTN64_R32", "ATTN64_R64", "ATTN128_R32", "ATTN128_R64", "ATTN128_R128_DEEP"}
DRIVER = r"""
#include <cstdio>
#include "attn_plan.hpp"
using namespace tp::k;
int main() {
  const int all[] = {NAMES};
  for (int i = 0; i < (int)(sizeof all / sizeof *all); ++i)
    if (all[i] != i) return 1;
  if (sizeof all / sizeof *all != ATTN_VARIANTS) return 2;
  long d, h, hk, b, nq, nk, causal, left, right, sinks;
  unsigned long scratch;
  while (std::scanf("%ld %ld %ld %ld %ld %ld %ld %ld %ld %ld %lu", &d, &h, &hk, &b, &nq, &nk, &causal, &left, &right, &sinks, &scratch) == 11) {
    const AttnPlan p = attn_plan((int)d, nq * (h / hk), hk * b, attn_span(nq, nk, causal != 0, left, right, sinks), scratch);
    std::printf("%d %d\n", p.variant, p.splits);
  }
}
"""
SCRATCH = 32 << 20


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    cxx = shutil.which("g++")
    if not cxx:
        pytest.skip("no C++ compiler")
    d = tmp_path_factory.mktemp("attn_plan")
    (d / "driver.cpp").write_text(DRIVER.replace("NAMES", ", ".join(KERNELS)))
    subprocess.run([cxx, "-O1", "-std=c++17", "-I", os.path.join(ROOT, "paper_2306_03622_amd", "csrc", "kernels"),
                    str(d / "driver.cpp"), "-o", str(d / "driver")], check=True)

    def run(calls):             # (dim, heads, kv_heads, batch, queries, keys, causal, left, right, sinks, scratch)
        out = subprocess.run([str(d / "driver")], input="\n".join(" ".join(str(int(v)) for v in c) for c in calls), check=True,
                             capture_output=True, text=True).stdout
        return [tuple(int(v) for v in line.split()) for line in out.splitlines()]

    return run


def test_the_gpu_shapes_reach_every_kernel(plan):
    calls = [(d, h, hk, b, nq, nk, kw.get("causal", False), *kw.get("window", (-1, -1)), kw.get("sinks", 0), SCRATCH if split else 0)
             for _, split, b, h, hk, d, nq, nk, kw in SHAPES]
    reached = set()
    for shape, (kernel, splits) in zip(SHAPES, plan(calls)):
        assert (KERNELS[kernel], splits > 1) == shape[:2], shape
        reached.add(shape[:2])
    assert reached == {(k, False) for k in KERNELS} | {(k, True) for k in SPLIT}


def test_plans_can_be_launched(plan):
    rng = random.Random(11)
    calls = []
    while len(calls) < 20000:
        hk = 2 ** rng.randint(0, 12) + rng.randint(0, 3)
        h, b = hk * rng.choice((1, 2, 3, 4, 8, 16)), 2 ** rng.randint(0, 16) + rng.randint(0, 3)
        nq, nk = 2 ** rng.randint(0, 24) + rng.randint(0, 3), 2 ** rng.randint(0, 29) + rng.randint(0, 3)
        if h > 65536 or nq * h * b >= 1 << 30 or b * hk >= 1 << 22:
            continue                                             # refused before
        left, right = (rng.choice((-1, 0, 2 ** rng.randint(0, 30) - 1)) for _ in range(2))
        calls.append((rng.choice((64, 128)), h, hk, b, nq, nk, rng.random() < 0.5, left, right, rng.choice((0, 4, 2 ** 31 - 1)),
                      rng.choice((0, 4096, SCRATCH, 2 ** 63))))
    most = (64, 1 << 14, 1 << 14, (1 << 8) - 1, 128, 1000, True, -1, -1, 0, SCRATCH)       # 2^22 key/value heads, nearly
    calls += [most, (128, *most[1:])]
    for c, (kernel, splits) in zip(calls, plan(calls)):
        d, h, hk, b, nq = c[:5]
        rows = nq * (h // hk)
        assert KERNELS[kernel].startswith(f"ATTN{d}_") and 1 <= splits <= 64
        assert -(-rows // ROWS[kernel]) * hk * b * splits * THREADS[kernel] < 2 ** 32, c
        assert splits == 1 or (splits * rows * hk * b * (d + 2) * 4 <= c[-1] and KERNELS[kernel] in SPLIT), c
