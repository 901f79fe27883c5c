// Which kernel a 4-bit linear layer takes (no HIP headers: also compiled for the host alone).
#pragma once
#include <cstdint>

namespace tp {
namespace k {

// Output features x rows a workgroup owns, sets of waves over the k-blocks (128 columns) of which each takes its share, its
// threads, and the time model's coefficients: us = launch + rounds (round + steps (step + group_step 128 / group)) + steps first, with
// `rounds` = workgroups / 256 CUs, rounded up, and `steps` = k-blocks a set takes.
struct W4Variant {
  int bn, bm, sets, threads;
  double launch, round, first, step, group_step;
};

enum { W4_ROWS16, W4_ROWS32, W4_ROWS64, W4_TILE32X32, W4_TILE64X32, W4_TILE64X32_DEEP, W4_TILE64X64, W4_TILE128X64,
       W4_TILE128X64_WIDE, W4_TILE256X128, W4_VARIANTS };

// Fitted to 2499 passes on MI355X (13 shapes from 96 x 200 to 8192 x 32768, the three groups, 1 to 5000 rows, graph replay,
// operands rotating beyond the L2s): choosing by the model costs 3% over the best variant of each case on average.
// What they trade, us, in groups of 128, of 4096 outputs and columns: 1 row ROWS16 4.9, ROWS64 7.9; 32 rows ROWS32 8.3, ROWS16 11.6;
// 64 rows ROWS64 9.7, ROWS32 13.9; 128 rows TILE64X32_DEEP 12.7, ROWS64 16.5; 256 rows TILE64X64 23.2, TILE64X32_DEEP 23.1 and 24.3;
// 1024 rows TILE128X64_WIDE 51.5, TILE64X64 61.9; 2048 rows TILE256X128 79, TILE128X64_WIDE 95 (in groups of 32 99 and 116); 8192 rows
// 312, 355. Of 4096 outputs and 768 columns: 24 rows ROWS16 4.2, ROWS32 4.4; 80 rows TILE64X32 5.3, ROWS64 6.2, TILE32X32 8.1. Of 768
// outputs and 4096 columns: 24 rows ROWS16 7.1, ROWS32 7.7, TILE32X32 8.7. The model counts rounds of 256 workgroups, though a CU holds
// up to three of the smaller tiles at a time: it expects 15.0 of 1024 x 2304 x 768, which takes 12.
constexpr W4Variant kW4[W4_VARIANTS] = {
    {16, 16, 4, 256, 2.565, 0.076, 0.0, 0.434, 0.055},    {32, 16, 8, 512, 2.405, 0.987, 0.0, 1.042, 0.069},
    {64, 16, 8, 512, 2.186, 0.465, 0.0, 1.445, 0.171},    {32, 32, 4, 512, 1.345, 2.383, 0.0, 0.689, 0.026},
    {64, 32, 2, 512, 2.676, 1.159, 0.132, 0.445, 0.027},  {64, 32, 4, 1024, 1.087, 3.302, 0.0, 0.945, 0.050},
    {64, 64, 1, 256, 3.160, 1.185, 0.203, 0.313, 0.039},  {128, 64, 1, 512, 1.658, 2.755, 0.213, 0.552, 0.061},
    {128, 64, 1, 256, 1.516, 3.731, 0.327, 0.439, 0.046}, {256, 128, 1, 512, 0.0, 7.269, 0.0, 1.727, 0.246}};

inline double w4_us(const W4Variant& v, int64_t M, int64_t N, int64_t K, int group) {
  const int64_t wgs = (N + v.bn - 1) / v.bn * ((M + v.bm - 1) / v.bm), kb = (K + 127) / 128;
  const double rounds = (double)((wgs + 255) / 256), steps = (double)((kb + v.sets - 1) / v.sets);
  return v.launch + rounds * (v.round + steps * (v.step + v.group_step * 128 / group)) + steps * v.first;
}

// Whether a variant can be launched: the kernels of few rows put their row tiles into a grid dimension of 65535 (from
// 1,048,561 rows on the tiles take over), the tiles are one grid of fewer than 2^32 threads.
inline bool w4_fits(int variant, int64_t M, int64_t N) {
  const W4Variant& v = kW4[variant];
  const int64_t tn = (N + v.bn - 1) / v.bn, tm = (M + v.bm - 1) / v.bm;
  return variant <= W4_ROWS64 ? tm <= 65535 : tn * tm * v.threads < 1ll << 32;
}

// The variant, or -1 where none can be launched: not while the rows in whole 128s times the features in whole 256s stay
// below 2^38, which the largest tiles take.
inline int w4_plan(int64_t M, int64_t N, int64_t K, int group) {
  int best = -1;
  double us = 0;
  for (int i = 0; i < W4_VARIANTS; ++i) {
    if (!w4_fits(i, M, N)) continue;
    // the largest tiles only where 16 k-blocks and more make up for the ring's filling, as the model does not see
    // (5000 rows, 1024 outputs, 256 columns: 16.0 us, TILE128X64 12.1), or where no others can be launched
    if (i == W4_TILE256X128 && K < 16 * 128 && best >= 0) continue;
    const double t = w4_us(kW4[i], M, N, K, group);
    if (best < 0 || t < us) {
      best = i;
      us = t;
    }
  }
  return best;
}

}  // namespace k
}  // namespace tp
