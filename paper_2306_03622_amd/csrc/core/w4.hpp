// 4-bit weights with group scales: sizes, the blocked order and quantisation (torpor_ops.h). Host-only C++.
#pragma once
#include <cstdint>

namespace tp {

inline bool w4_shape_ok(int64_t N, int64_t K, int64_t group) {
  return N >= 1 && N <= (1 << 24) && K >= 1 && K <= (1 << 20) && (group == 32 || group == 64 || group == 128) &&
         K % group == 0;
}

inline uint64_t w4_code_bytes(int64_t N, int64_t K) { return (uint64_t)((N + 15) / 16) * ((K + 127) / 128) * 1024; }
inline uint64_t w4_scale_bytes(int64_t N, int64_t K, int64_t group) {
  return (uint64_t)((N + 15) / 16) * ((K + 127) / 128) * (128 / group) * 32;
}

// Plain order (codes [N][K/2], scales [N][K/group]) to blocked order; the shape passes w4_shape_ok.
void w4_pack_codes(const uint8_t* codes, int64_t N, int64_t K, uint8_t* out);
void w4_pack_scales(const uint16_t* scales, int64_t N, int64_t K, int64_t group, uint16_t* out);

// Rounds w[N][K] to the plain order; false if a group's scale would not be finite.
bool w4_quantize(const float* w, int64_t N, int64_t K, int64_t group, uint8_t* codes, uint16_t* scales);

}  // namespace tp
