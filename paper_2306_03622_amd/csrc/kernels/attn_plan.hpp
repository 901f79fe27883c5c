// Which kernel a call of the masked attention takes, and over how many workgroups its keys are split (no HIP headers: also
// compiled for the host alone).
#pragma once
#include <algorithm>
#include <cstdint>

namespace tp {
namespace k {

// Kernels: head dim, 32-row waves side by side, waves deep over the keys, 32-key blocks a wave, stages in LDS (attn_masked.hip)
enum {
  ATTN64_R32, ATTN64_R64, ATTN64_R128, ATTN64_R128_LONG, ATTN128_R32, ATTN128_R64, ATTN128_R128_DEEP, ATTN128_R128, ATTN128_R256,
  ATTN_VARIANTS
};

struct AttnPlan {
  int variant, splits;
};

// Keys that a workgroup walks, about. left, right: the window, negative: none.
inline int64_t attn_span(int64_t q_len, int64_t kv_len, bool causal, int64_t left, int64_t right, int64_t sinks) {
  if (left < 0 || (!causal && right < 0)) return kv_len;
  return std::min<int64_t>(kv_len, left + (causal ? 0 : right) + std::min<int64_t>(q_len, 128) + sinks);
}

// rows: q_len times the query heads of a key/value head; heads: key/value heads of all sequences; scratch: bytes for the splits'
// partial results.
inline AttnPlan attn_plan(int dim, int64_t rows, int64_t heads, int64_t span, uint64_t scratch) {
  auto wgs = [&](int64_t r) { return (rows + r - 1) / r * heads; };      // workgroups of r rows
  // Splits of the keys over workgroups, to 256 of them, of at least three tiles of kt keys, as far as the scratch holds them (a
  // lane of the joining wave for each). One token, 8 / 1 heads of 128 over 30,000 keys: 64 splits 17.9 us, 32 19.4, 16 25.2, none 240;
  // 32 / 8 over 8000: 20 splits 16.2, 8 18.4; 8 x 32 / 8 over 3000: 8 splits 24.0, 16 27.7; ten over 600, 12 of 64: none 7.5, four 9.2.
  auto splits = [&](int64_t workgroups, int kt) {
    const int64_t fits = (int64_t)(scratch / 4) / (rows * heads * (dim + 2));
    return (int)std::max<int64_t>(1, std::min<int64_t>({256 / workgroups, span / (3 * kt), 64, fits}));
  };
  // Measured on MI355X (us), heads / key/value heads x dim, queries over keys:
  //   32 rows, four waves deep: few tokens, whose cost is the latency, and short sequences that would not give every CU a larger tile:
  //     32 / 8 x 128, 8 over 8000 24.5 (64 rows 28.1), 20 over 8000 22.6 (128 rows 31.1), 8 / 1, 1 over 30,000 29.4 (64
  //     rows 31.7); 12 x 64, 5 x 96 5.3 (5.6), 512 over 512 7.4 (12.6).
  //   64 rows, two deep, one tile more under way: tokens whose cost is the memory's: 32 / 8 x 128, 1 over 100,001 92.6 (32 rows 97.3), 16 x 1
  //     with a window of 1024 19.9 (21.1); 12 x 64, 16 x 1 over 3000 36.6 (42.7). Also 32 / 8 x 128, 500 over 500 13.0 (128 rows, two
  //     deep 22.1); at dim 64 up to four on every CU: 12 x 64, 8 x 512 16.9 (128 rows 18.2), 4096 with a window of 256 19.0 (22.6).
  //   128 rows, two deep, 64 keys a wave, at dim 128 up to one on every CU: 32 / 8, 2 x 500 over 6000 with a window of 1024 30.8 (one deep
  //     34.4), 100 over 5000 24.8 (29.0). But 32 / 32, 2 x 1000 53.1 (one deep 44.3).
  //   256 rows for long walks at dim 128, two on every CU and more: 32 / 8, 4096 causal 150 (128 rows 158), 8191 552 (559).
  //   128 rows else: 32 / 8 x 128, 4 x 2000 with a window of 512 99 (256 rows 110); 12 x 64, 8 x 2048 with
  //     a window of 128 34.5 (64 rows 45). There 32 keys a wave, but 64 on long walks: 8000 causal 153 (32 keys 168), 4 x 2048 78 (85);
  //     with the window 36.
  const bool d64 = dim == 64, heavy = heads * span * dim >= 1 << 24;
  if ((rows <= (d64 ? 64 : 128) && !heavy) || (rows > 64 && wgs(32) <= 256 && span <= 1024))
    return {d64 ? ATTN64_R32 : ATTN128_R32, splits(wgs(32), 128)};
  if (rows <= 64 || (d64 ? wgs(64) <= 1024 : wgs(64) <= 256 && span <= 1024))
    return {d64 ? ATTN64_R64 : ATTN128_R64, splits(wgs(64), 64)};
  if (!d64 && wgs(128) <= 256) return {ATTN128_R128_DEEP, splits(wgs(128), 128)};
  if (d64) return {span >= 1024 ? ATTN64_R128_LONG : ATTN64_R128, 1};
  return {span >= 2048 && wgs(256) >= 512 ? ATTN128_R256 : ATTN128_R128, 1};
}

}  // namespace k
}  // namespace tp
