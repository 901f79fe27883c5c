// Host work in parts, a thread each.
#pragma once
#include <thread>

namespace tp {

constexpr int kMostParts = 8;

// f(0) .. f(n - 1), n <= kMostParts, f throws nothing: all done on return. A part that no thread can be started for (which
// throws, at a C entry that must not) runs here.
template <typename F>
void in_parts(int n, const F& f) {
  std::thread th[kMostParts];
  for (int i = 0; i < n; ++i) {
    try {
      th[i] = std::thread([&f, i] { f(i); });
    } catch (...) {
      f(i);
    }
  }
  for (int i = 0; i < n; ++i)
    if (th[i].joinable()) th[i].join();
}

}  // namespace tp
