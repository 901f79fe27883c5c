"""Host work in parts (packing of a model's weights at registration): every part is done, also where no thread can be started."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
DRIVER = r"""
#include <sys/resource.h>
#include <unistd.h>
#include <atomic>
#include <cstdio>
#include <cstdlib>
#include "core/parts.hpp"
static long pages() {
  long n = 0;
  if (FILE* f = std::fopen("/proc/self/statm", "r")) {
    if (std::fscanf(f, "%ld", &n) != 1) n = 0;
    std::fclose(f);
  }
  return n;
}
static bool run() {
  for (int n = 0; n <= tp::kMostParts; ++n) {
    std::atomic<int> done[tp::kMostParts] = {};
    tp::in_parts(n, [&](int i) { ++done[i]; });
    for (int i = 0; i < tp::kMostParts; ++i)
      if (done[i] != (i < n)) return false;
  }
  return true;
}
int main() {
  if (!run()) return 1;
  // no address space for another thread's stack
  const rlim_t now = (rlim_t)pages() * 4096 + (1 << 20);
  const rlimit lim{now, now};
  if (setrlimit(RLIMIT_AS, &lim) != 0) return 2;
  int started = 0;
  for (int i = 0; i < 64; ++i) {           // (stacks of threads that have ended are used again: take those first)
    try {
      std::thread* t = new std::thread([&] { for (;;) pause(); });
      t->detach();
      ++started;
    } catch (...) {
      break;
    }
  }
  if (started == 64) return 3;
  const bool ok = run();
  std::_Exit(ok ? 0 : 4);
}
"""


def test_parts_are_done_with_threads_and_without(tmp_path):
    cxx = shutil.which("g++")
    if not cxx:
        pytest.skip("no C++ compiler")
    (tmp_path / "d.cpp").write_text(DRIVER)
    subprocess.run([cxx, "-O1", "-std=c++17", "-pthread", "-I", os.path.join(ROOT, "paper_2306_03622_amd", "csrc"), str(tmp_path / "d.cpp"),
                    "-o", str(tmp_path / "d")], check=True)
    r = subprocess.run([str(tmp_path / "d")], timeout=60)
    assert r.returncode == 0
