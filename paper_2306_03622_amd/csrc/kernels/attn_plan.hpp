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
  // lane of the joining wave for each). One token, 8 / 1 heads of 128 over 30,000 keys: 64 splits 18.7 us, 32 19.9, 16 25.4, none 241;
  // 32 / 8 over 8000: 20 splits 16.8, 8 18.7; 8 x 32 / 8 over 3000: four splits 24.8, two 31.9, eight 28.5; ten over 600, 12 of 64: none
  // 7.6, four 8.8. From 129 workgroups on there is one walk for each, so that up to 511 some
  // CUs have more to do than others: one token of 16 / 17 / 32 / 33 sequences, 32 / 8 over 4096, 55 / 69 / 97 / 149.
  auto splits = [&](int64_t workgroups, int kt) {
    const int64_t fits = (int64_t)(scratch / 4) / (rows * heads * (dim + 2));
    return (int)std::max<int64_t>(1, std::min<int64_t>({256 / workgroups, span / (3 * kt), 64, fits}));
  };
  // Measured on MI355X (us, graph replay), heads / key/value heads x dim, queries over keys:
  //   32 rows, four waves deep: few tokens, whose cost is the latency, and short sequences that would not give every CU a larger tile:
  //     8 / 1 x 128, 1 over 30,000 18.7 (64 rows 20.0); 12 x 64, 5 x 96 5.5 (5.9), 512 over 512 7.6 (13.3). Not faster for a few tokens over a
  //     longer cache: 32 / 8 x 128, 8 over 8000 17.6 (64 rows 16.3), 20 over 8000 19.2 (64 rows 17.9, 128 rows 20.9).
  //   64 rows, two deep, one tile more under way: tokens whose cost is the memory's: 32 / 8 x 128, 1 over 100,001 80.5 (32 rows 84.7), 16 x 1
  //     with a window of 1024 20.5 (22.2); 12 x 64, 16 x 1 over 3000 37.2 (43.1). Also 32 / 8 x 128, 500 over 500 12.7 (32 rows 16.8, 128 rows
  //     15.5); at dim 64 up to four on every CU: 12 x 64, 8 x 512 15.3 (128 rows 15.4 to 16.9), 4096 with a window of 256 19.7 (22.6).
  //   128 rows, two deep, 64 keys a wave, at dim 128 up to one on every CU: 32 / 8, 2 x 500 over 6000 with a window of 1024 31.4 (one deep
  //     32.1, 64 rows 43.1), 100 over 5000 25.2 (28.2 with 64 rows, one deep and unsplit 99). Beyond one deep: 32 / 32, 2 x 1000 32.8 (two deep 36.1).
  //   256 rows for long walks at dim 128, two on every CU and more: 32 / 8, 4096 causal 154 (128 rows 166), 8191 575 (588).
  //   128 rows else: 32 / 8 x 128, 4 x 2000 with a window of 512 87 (256 rows 95); 12 x 64, 8 x 2048 with
  //     a window of 128 31.6 (64 rows 37.9). There 32 keys a wave, but 64 on long walks: 8000 causal 154 (32 keys 169), 4 x 2048 72.4 (76.7);
  //     with the window 32.7.
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
