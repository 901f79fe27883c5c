// How a call of the attention over a paged cache is split (no HIP headers: also compiled for the host alone).
#pragma once
#include <algorithm>
#include <cstdint>

namespace tp {
namespace k {

struct CachePlan {
  int rb, splits;         // blocks of 16 rows a workgroup takes, workgroups over the keys
};

// Keys that a workgroup walks, about. window: negative: none.
inline int64_t cache_span(int64_t q_len, int64_t kv_len, int64_t window, int64_t sinks) {
  return window < 0 ? kv_len : std::min<int64_t>(kv_len, window + std::min<int64_t>(q_len, 64) + sinks);
}

// rows: q_len times the query heads of a key/value head; heads: key/value heads of all sequences; scratch: bytes for the splits'
// partial results.
inline CachePlan cache_plan(int dim, bool e4m3, int64_t rows, int64_t heads, int64_t span, uint64_t scratch) {
  (void)e4m3;
  const int rb = rows <= 16 ? 1 : rows <= 32 ? 2 : 4;
  const int64_t wgs = (rows + 16 * rb - 1) / (16 * rb) * heads;
  const int64_t fits = (int64_t)(scratch / 4) / (rows * heads * (dim + 2));
  return {rb, (int)std::max<int64_t>(1, std::min<int64_t>({512 / wgs, span / 256, 64, fits}))};
}

}  // namespace k
}  // namespace tp
