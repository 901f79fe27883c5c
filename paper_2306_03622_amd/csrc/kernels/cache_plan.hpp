// How calls on a paged cache, rows in and out of it and attention over it, are split (no HIP headers: also compiled for the host alone).
#pragma once
#include <algorithm>
#include <cstdint>

namespace tp {
namespace k {

struct CacheRowsPlan {
  int per, cols;          // lanes that a token takes, workgroups of 256 side by side for one (more than 1: then a row at a time)
  int rows, each;         // rows side by side in a workgroup, rows in each place
  int64_t blocks;         // workgroups along a sequence's rows
};

// heads: key/value heads; q_len: rows of each of `batch` sequences.
inline CacheRowsPlan cache_rows_plan(int dim, int64_t heads, int64_t batch, int64_t q_len) {
  CacheRowsPlan p{};
  p.per = (int)heads * (dim / 8);
  p.cols = (p.per + 255) / 256;
  p.rows = p.cols > 1 ? 1 : 256 / p.per;
  // two rows in each place where that still gives every CU two workgroups (two prompts of 3001 in 8 bits 8.8 us, with four 9.8, one 9.4)
  auto blocks = [&](int64_t each) { return (q_len + p.rows * each - 1) / (p.rows * each); };
  p.each = blocks(2) * p.cols * batch >= 512 ? 2 : 1;
  p.blocks = blocks(p.each);
  return p;
}

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
  // one wave where the keys are two tiles at most (us, graph replay: 25 sequences of 12 key/value heads, up to 8 tokens 5.8, four waves 11.4)
  if (rb == 1 && span <= 64) return {1, 1, 1};
  const int64_t fits = (int64_t)(scratch / 4) / (rows * heads * (dim + 2));
  const int64_t most = std::max<int64_t>(1, std::min<int64_t>({64, span / 128, fits, ((1 << 24) - 1) / wgs}));       // grids below 2^32 lanes
  // (Times here with exponentials in one part; the second adds 1 to 4% to both sides.) Time by a model, in ns and bytes: a workgroup takes 3500 beside its keys, which come at 5400 for all, at most 7.5 (8 bits: 5.5) for
  // a wave; on a CU run as many workgroups as its LDS holds. Where lengths differ they are taken to be three quarters of the longest on
  // average, short ones making room for the next. Partial results are written and read at 5000, and joined in 3000. Of 20 shapes the
  // choice was within 7% of the best of 22. Two waves instead of four (us): 32 / 8 heads of 128, 64 sequences of up to 128 / 256 / 500
  // tokens 7.7 / 11.9 / 19.8 instead of 12.1 / 16.9 / 23.8, 8 of up to 300 8.5 instead of 6.9.
  const double bytes = (double)span * 2 * dim * (e4m3 ? 1 : 2), part = (double)rows * heads * (dim + 2) * 8;
  const int64_t ring = 64 * dim * (e4m3 ? 1 : 2) * (dim == 64 ? 3 : 2);       // a wave's (the exponents aside)
  CachePlan best{rb, 4, 1};
  double least = 0;
  for (int waves = 4; waves >= (rb == 1 ? 2 : 4); waves -= 2) {
    const int64_t once = 256 * std::max<int64_t>(1, 160 * 1024 / (ring * waves + 1024));
    for (int64_t s = 1; s <= most; ++s) {
      const int64_t n = wgs * s;
      const double one = waves * (e4m3 ? 5.5 : 7.5), each = bytes / s / std::min(one, 5400.0 / (double)std::min<int64_t>(once, n));
      const double rounds = (double)((n + once - 1) / once);
      double t = rounds * (3500 + each);
      if (!even) t = std::max(3500 + bytes / s / one, rounds * 3500 + 0.75 * bytes * wgs / 5400 + 0.25 * each);
      if (s > 1) t += 3000 + part * s / 5000;
      if (least == 0 || t < least) least = t, best = {rb, waves, (int)s};
    }
  }
  return best;
}

}  // namespace k
}  // namespace tp
