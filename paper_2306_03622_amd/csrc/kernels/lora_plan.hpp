// How a call of the low-rank adapters is split (no HIP headers: also compiled for the host alone).
#pragma once
#include <algorithm>
#include <cstdint>

namespace tp {
namespace k {

constexpr int kLoraRank = 128;          // the largest rank
constexpr int kLoraFew = 7;             // adapters whose rows are put in order beside the first product,
constexpr int kLoraFewRows = 1 << 14;   // and rows

struct LoraPlan {
  int splits;             // workgroups along K; 0: both products in one launch, no scratch
  int tall;               // tiles of 64 rows, first product, else of 32
  int down_slots;         // workgroups that share the adapters of such a tile
  int up_slots;           // and of a tile of 64 rows, second product
  int run;                // blocks of 64 outputs a workgroup, second product
  int order;              // rows adapter by adapter: 0 not, 1 first, 2 beside the first product, for the second
};

inline LoraPlan lora_plan(int64_t M, int64_t N, int64_t K, int64_t R, int64_t adapters, uint64_t scratch) {
  const int64_t fits = (int64_t)(scratch / 4) / (M * R);
  if (fits < 1 || M >= 1 << 27) return {0, 0, 0, 0, 0, 0};
  // One adapter, small: in one launch (us, graph replay, one / two launches): 1 row of 768 x 768, rank 8 5.1 / 6.7, rank 64 9.0 / 8.7; 1 of
  // 4096 x 4096, rank 16 10.1 / 7.8; 256 of 256 x 256, rank 8 5.6 / 7.7. Adapters of one tile come one after the other
  // there: 64 rows of 8, 768 x 768, rank 8 26 / 8.5.
  if (std::min(M, adapters) == 1 && K * ((R + 15) / 16) <= 2048 && M <= 256) return {0, 0, 0, 0, 0, 0};
  // Tall tiles read A half as often, at ranks where that is most of what a CU reads: five adapters of 64, 8192 rows of 4096 20 us, else 25.
  const bool tall = R > 32 && R <= 64 && M >= 4096 && K >= 1024;
  const int64_t tiles = tall ? (M + 63) / 64 : (M + 31) / 32, blocks = (N + 63) / 64, jobs = (M + 63) / 64;
  // Beside the first product: hidden by it where K is long, lost where rows are in order anyway and it is short (us, without / with:
  // 8192 rows of 4096 x 4096, rank 64, five adapters in turn 153 / 77, one after the other 70 / 70; 2048 of 768 x 3008, rank 8, seven in turn
  // 29 / 15; 8192 of 512 x 512, rank 16, seven in turn 27 / 19, one after the other 15.7 / 19.7; 16000 of 512 x 1024 so 27 / 38).
  const bool holds = (int64_t)(scratch / 4) >= M * (R + 2);
  const bool many = adapters >= 8 && adapters < 4096 && M > 128 && M <= 1 << 17 && M * std::min<int64_t>(adapters, 64) >= 8192;
  const bool few = adapters >= 2 && adapters <= kLoraFew && M >= 512 && M <= kLoraFewRows && K >= 512 && M <= 16 * K;
  const int order = !holds ? 0 : many ? 1 : few ? 2 : 0;
  // adapters of a tile: in order few, and two slots for tiles where one adapter's rows end and another's begin
  const int64_t kinds = order ? std::min<int64_t>(adapters, 1 + (adapters + jobs - 1) / jobs) : adapters;
  const int64_t room = order ? (int64_t)((scratch / 4 - 2 * M) / (M * R)) : fits;
  const int64_t ds = std::max<int64_t>(1, std::min<int64_t>({order == 1 ? kinds : adapters, 32, M, std::max<int64_t>(2, 512 / tiles)}));
  const int64_t z = std::max<int64_t>(1, std::min<int64_t>({K / 512, 8, 512 / (tiles * ds), room}));
  const int64_t us = std::max<int64_t>(1, std::min<int64_t>({kinds, 64, M, std::max<int64_t>(2, 4096 / (jobs * blocks))}));
  const int64_t run = std::max<int64_t>(1, std::min<int64_t>(8, (jobs * blocks * us + 767) / 768));
  return {(int)z, tall, (int)ds, (int)us, (int)run, order};
}

// Rows that are taken at once: all of them where scratch holds their inner sums (and their order, where they are put in one), else
// parts one after the other, each with launches of its own: multiples of 64 rows, as few and as even as the scratch allows. Parts have 1024 rows at
// least, and 4096 where one launch computes the inner sums once; below, everything goes in one launch. us, graph replay, one launch / parts of
// 512 / 1024 / 4096 rows: 4096 rows of 4096 x 4096, 32 adapters of rank 16 2028 / 140 / 77 / 32, 16384 of 2048 x 2048, four of 32 806 / 318 / 210 / 95, 4096 of
// 256 -> 4096, one of 16 34 / 73 / 44 / 22, 1024 -> 1024, one of 64 38 / 91 / 46 / 20; to 256 outputs: 4096 of 4096, one of 64
// 55 / 117 / 61 / 23, 16384 of 1024, four of 64 133 / 347 / 176 / 68.
inline int64_t lora_rows(int64_t M, int64_t N, int64_t K, int64_t R, int64_t adapters, uint64_t scratch) {
  const int64_t words = (int64_t)(scratch / 4), least = N <= 256 ? 4096 : 1024;
  const int64_t most = std::min<int64_t>(words / (R + 2), (1 << 27) - 1) / 64 * 64;        // (a call in two launches has fewer than 2^27 rows)
  if (most < least || (M <= words / (R + 2) && M < 1 << 27)) return M;
  if (M <= words / R && M < 1 << 27 && lora_plan(M, N, K, R, adapters, ~0ull >> 1).order == 0) return M;
  const int64_t parts = (M + most - 1) / most, rows = (M + parts - 1) / parts;
  return std::max(least, (rows + 63) / 64 * 64);
}

}  // namespace k
}  // namespace tp
