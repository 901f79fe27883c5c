// How a call of the low-rank adapters is split (no HIP headers: also compiled for the host alone).
#pragma once
#include <algorithm>
#include <cstdint>

namespace tp {
namespace k {

constexpr int kLoraRank = 128;          // the largest rank

struct LoraPlan {
  int splits;             // workgroups along K; 0: both products in one launch, no scratch
  int down_slots;         // workgroups that share the adapters of a tile of 32 rows, first product
  int up_slots;           // and of 64 rows, second product
};

inline LoraPlan lora_plan(int64_t M, int64_t N, int64_t K, int64_t R, int64_t adapters, uint64_t scratch) {
  const int64_t fits = (int64_t)(scratch / 4) / (M * R);
  if (fits < 1 || M >= 1 << 27) return {0, 0, 0};
  const int64_t tiles = (M + 31) / 32;
  const int64_t ds = std::max<int64_t>(1, std::min<int64_t>({adapters, 32, M, 512 / tiles}));
  const int64_t z = std::max<int64_t>(1, std::min<int64_t>({K / 1024, 8, 512 / (tiles * ds), fits}));
  const int64_t wgs = (M + 63) / 64 * ((N + 255) / 256);
  const int64_t us = std::max<int64_t>(1, std::min<int64_t>({adapters, 64, M, 2048 / wgs}));
  return {(int)z, (int)ds, (int)us};
}

}  // namespace k
}  // namespace tp
