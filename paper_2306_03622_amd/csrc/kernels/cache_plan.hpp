// How a call of the attention over a paged cache is split (no HIP headers: also compiled for the host alone).
#pragma once
#include <algorithm>
#include <cstdint>

namespace tp {
namespace k {

struct CachePlan {
  int rb, waves, splits;  // blocks of 16 rows a workgroup takes, its waves over the keys, workgroups over the keys
};

// Keys that a workgroup walks, about. window: negative: none.
inline int64_t cache_span(int64_t q_len, int64_t kv_len, int64_t window, int64_t sinks) {
  return window < 0 ? kv_len : std::min<int64_t>(kv_len, window + std::min<int64_t>(q_len, 64) + sinks);
}

// rows: q_len times the query heads of a key/value head; heads: key/value heads of all sequences; even: sequences walk about as many
// keys each; scratch: bytes for the splits' partial results.
inline CachePlan cache_plan(int dim, bool e4m3, int64_t rows, int64_t heads, int64_t span, bool even, uint64_t scratch) {
  const int rb = rows <= 16 ? 1 : rows <= 32 ? 2 : 4;
  const int64_t wgs = (rows + 16 * rb - 1) / (16 * rb) * heads;
  const int64_t fits = (int64_t)(scratch / 4) / (rows * heads * (dim + 2));
  const int64_t most = std::min<int64_t>({64, span / 128, fits});
  // Time by a model, in ns and bytes: a workgroup takes 3500 beside its keys, which come at 5400 for all, at most 30 (8 bits: 22) for one;
  // 256 (8 bits: 512) run at once. Where lengths differ they are taken to be three quarters of the longest on average, short ones making
  // room for the next. Partial results are written and read at 5000, and joined in 3000.
  const double bytes = (double)span * 2 * dim * (e4m3 ? 1 : 2), part = (double)rows * heads * (dim + 2) * 8, one = e4m3 ? 22 : 30;
  const int64_t once = e4m3 ? 512 : 256;
  double best = 0;
  int splits = 1;
  for (int64_t s = 1; s <= std::max<int64_t>(1, most); ++s) {
    const int64_t n = wgs * s;
    const double each = bytes / s / std::min(one, 5400.0 / (double)std::min<int64_t>(once, n));
    const double rounds = (double)((n + once - 1) / once);
    double t = rounds * (3500 + each);
    if (!even) t = std::max(3500 + bytes / s / one, rounds * 3500 + 0.75 * bytes * wgs / 5400 + 0.25 * each);
    if (s > 1) t += 3000 + part * s / 5000;
    if (s == 1 || t < best) best = t, splits = (int)s;
  }
  return {rb, rb == 1 && span <= 64 ? 1 : 4, splits};
}

}  // namespace k
}  // namespace tp
