"""The plans of the serving operators (host code, compiled here): the GPU tests' shapes reach every kernel, and every call within the
documented sizes gets grids that can be launched and partial results that its scratch holds."""
import os
import random
import shutil
import subprocess

import pytest

from tests.test_gpu_serve_variants import ATTENTION, LORA, PAIRS

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
DRIVER = r"""
#include <cstdio>
#include "cache_plan.hpp"
#include "lora_plan.hpp"
using namespace tp::k;
int main() {
  char what;
  long a, b, c, d, e, f, g, h, i;
  unsigned long scratch;
  while (std::scanf(" %c", &what) == 1)
    if (what == 'c') {          // dim, e4m3, heads, key/value heads, batch, queries, keys, window, sinks, scratch
      if (std::scanf("%ld %ld %ld %ld %ld %ld %ld %ld %ld %lu", &a, &b, &c, &d, &e, &f, &g, &h, &i, &scratch) != 10) return 1;
      const long span = cache_span(f, g, h, i);
      const CachePlan p = cache_plan((int)a, b != 0, f * (c / d), d * e, span, e == 1 || span <= g / 2, scratch);
      std::printf("%d %d %d\n", p.rb, p.waves, p.splits);
    } else {                    // rows, outputs, inputs, rank, adapters, scratch
      if (std::scanf("%ld %ld %ld %ld %ld %lu", &a, &b, &c, &d, &e, &scratch) != 6) return 1;
      const LoraPlan p = lora_plan(a, b, c, d, e, scratch);
      std::printf("%d %d %d %d %d %d\n", p.splits, p.tall, p.down_slots, p.up_slots, p.run, (int)p.order);
    }
}
"""
SCRATCH = 32 << 20


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    cxx = shutil.which("g++")
    if not cxx:
        pytest.skip("no C++ compiler")
    d = tmp_path_factory.mktemp("serve_plan")
    (d / "driver.cpp").write_text(DRIVER)
    subprocess.run([cxx, "-O1", "-std=c++17", "-I", os.path.join(ROOT, "paper_2306_03622_amd", "csrc", "kernels"),
                    str(d / "driver.cpp"), "-o", str(d / "driver")], check=True)

    def run(what, calls):
        out = subprocess.run([str(d / "driver")], input="\n".join(what + " " + " ".join(str(int(v)) for v in c) for c in calls),
                             check=True, capture_output=True, text=True).stdout
        return [tuple(int(v) for v in line.split()) for line in out.splitlines()]

    return run


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("dim", [64, 128])
def test_the_gpu_shapes_reach_every_attention_kernel(plan, dim, e4m3):
    calls, shapes = [], ATTENTION + PAIRS[dim, e4m3]
    for _, nq, h, hk, page, lens, kw in shapes:
        room = max((n + page - 1) // page for n in lens) * page
        calls.append((dim, e4m3, h, hk, len(lens), nq, room, kw.get("window", -1), kw.get("sinks", 0), SCRATCH))
    reached = set()
    for shape, (rb, waves, splits) in zip(shapes, plan("c", calls)):
        assert (rb, waves, splits > 1) == shape[0], (shape, splits)
        reached.add(shape[0])
    assert reached >= {(1, 1, False), (1, 2, False), *((rb, 4, s) for rb in (1, 2, 4) for s in (False, True))}


def test_the_gpu_shapes_reach_every_adapter_kernel(plan):
    calls = [(m, n, k, r, slots, SCRATCH) for _, m, k, n, r, slots, _ in LORA]
    reached = set()
    for shape, (splits, tall, _, _, run, order) in zip(LORA, plan("l", calls)):
        r = shape[4]
        rb, rc = ((r + 15) // 16, (r + 31) // 32)
        rb, rc = (rb if rb < 3 else 4 if rb < 5 else 8), (rc if rc < 3 else 4)
        assert (rb, rc, splits, run > 1, order) == shape[0], (shape, splits, run, order)
        reached |= {("down", rb), ("tall", bool(tall)), ("up", rc), ("order", order), ("run", run > 1)} if splits else {("one",)}
    assert reached == {("one",), *(("down", i) for i in (1, 2, 4, 8)), *(("up", i) for i in (1, 2, 4)),
                       *(("order", i) for i in (0, 1, 2)),
                       *((w, b) for w in ("tall", "run") for b in (False, True))}


def test_attention_plans_can_be_launched(plan):
    rng = random.Random(12)
    calls = [(d, e, 1 << 14, 1 << 14, 255, 8, 10 ** 6, -1, 0, SCRATCH) for d in (64, 128) for e in (0, 1)]     # the most key/value heads
    while len(calls) < 20000:
        hk = 2 ** rng.randint(0, 12) + rng.randint(0, 3)
        h, b = hk * rng.choice((1, 2, 3, 4, 8, 16, 40)), 2 ** rng.randint(0, 16) + rng.randint(0, 3)
        nq, nk = 2 ** rng.randint(0, 20) + rng.randint(0, 3), 2 ** rng.randint(0, 29) + rng.randint(0, 3)
        if h > 65536 or nq * h * b >= 1 << 27 or b * hk >= 1 << 22:
            continue                                             # refused before
        calls.append((rng.choice((64, 128)), rng.random() < 0.5, h, hk, b, nq, rng.choice((0, nk)), rng.choice((-1, 0, 2 ** rng.randint(0, 30) - 1)),
                      rng.choice((0, 4, 2 ** 31 - 1)), rng.choice((0, 4096, SCRATCH, 2 ** 63))))
    for c, (rb, waves, splits) in zip(calls, plan("c", calls)):
        d, _, h, hk, b, nq = c[:6]
        rows = nq * (h // hk)
        assert (rb, waves) in {(1, 1), (1, 2), (1, 4), (2, 4), (4, 4)} and 1 <= splits <= 64
        assert rows <= 16 * rb or rb == 4
        assert -(-rows // (16 * rb)) * hk * b * splits * waves * 64 < 2 ** 32, c
        assert splits == 1 or splits * rows * hk * b * (d + 2) * 4 <= c[-1], c


def test_adapter_plans_can_be_launched(plan):
    rng = random.Random(13)
    calls = []
    while len(calls) < 20000:
        m, n = (min(2 ** 31 - 1, 2 ** rng.randint(0, 31) + rng.randint(0, 9)) for _ in range(2))
        if (m + 15) // 16 * ((n + 255) // 256) >= 1 << 24:
            continue                                             # refused before
        calls.append((m, n, 8 * rng.choice((1, 3, 2 ** rng.randint(0, 17))), 8 * rng.randint(1, 16), rng.choice((1, 2, 5, 8, 100, 5000, 10 ** 6)),
                      rng.choice((0, 4096, SCRATCH, 2 ** 40, 2 ** 63))))
    for c, (splits, tall, ds, us, run, order) in zip(calls, plan("l", calls)):
        m, n, _, r, adapters, scratch = c
        if splits == 0:
            continue                                             # (m + 15) / 16 times (n + 255) / 256 workgroups of 256
        assert splits >= 1 and ds >= 1 and us >= 1 and 1 <= run <= 8
        assert ((m + 31) // 32 * ds * splits + (order == 2)) * 256 < 2 ** 32 and (not tall or 32 < r <= 64), c
        tiles = (m + 63) // 64
        assert (tiles if tiles < 8 else (tiles + 7) // 8 * 8) * us * -(-(-(-n // 64)) // run) * 256 < 2 ** 32, c
        assert 4 * m * (splits * r + (2 if order else 0)) <= scratch, c
        assert adapters < 4096 if order == 1 else 2 <= adapters <= 7 if order else True
