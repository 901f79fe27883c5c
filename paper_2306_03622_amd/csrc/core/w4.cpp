#include "w4.hpp"

#include <algorithm>
#include <cmath>
#include <cstring>

#include "errors.hpp"
#include "torpor_ops.h"

namespace tp {

namespace {

// fp32 -> bf16 bits, round to nearest even (finite values)
uint16_t bf16_bits(float f) {
  uint32_t u;
  std::memcpy(&u, &f, 4);
  return (uint16_t)((u + 0x7fffu + ((u >> 16) & 1)) >> 16);
}

float bf16_value(uint16_t b) {
  const uint32_t u = (uint32_t)b << 16;
  float f;
  std::memcpy(&f, &u, 4);
  return f;
}

}  // namespace

void w4_pack_codes(const uint8_t* codes, int64_t N, int64_t K, uint8_t* out) {
  const int64_t nb = (N + 15) / 16, kb = (K + 127) / 128;
  for (int64_t i = 0; i < nb; ++i)
    for (int64_t j = 0; j < kb; ++j)
      for (int q = 0; q < 4; ++q)
        for (int r = 0; r < 16; ++r)
          for (int t = 0; t < 4; ++t) {
            const int64_t row = 16 * i + r, col = 128 * j + 32 * t + 8 * q;
            uint32_t word = 0x88888888u;                  // 8 columns are padding together: K % 32 == 0
            if (row < N && col < K) {
              const uint8_t* src = codes + row * (K / 2) + col / 2;
              word = 0;
              for (int p = 0; p < 4; ++p)                 // columns 2 p and 2 p + 1 of the eight
                word |= (uint32_t)(src[p] & 15) << (4 * p) | (uint32_t)(src[p] >> 4) << (4 * p + 16);
            }
            uint8_t* d = out + ((i * kb + j) * 256 + 4 * (16 * q + r) + t) * 4;
            for (int b = 0; b < 4; ++b) d[b] = (uint8_t)(word >> (8 * b));
          }
}

void w4_pack_scales(const uint16_t* scales, int64_t N, int64_t K, int64_t group, uint16_t* out) {
  const int64_t nb = (N + 15) / 16, ng = (K + 127) / 128 * (128 / group), have = K / group;
  for (int64_t i = 0; i < nb; ++i)
    for (int64_t g = 0; g < ng; ++g)
      for (int r = 0; r < 16; ++r) {
        const int64_t row = 16 * i + r;
        out[(i * ng + g) * 16 + r] = row < N && g < have ? scales[row * have + g] : (uint16_t)0;
      }
}

bool w4_quantize(const float* w, int64_t N, int64_t K, int64_t group, uint8_t* codes, uint16_t* scales) {
  for (int64_t n = 0; n < N; ++n)
    for (int64_t g = 0; g < K / group; ++g) {
      const float* v = w + n * K + g * group;
      float top = 0.f;
      for (int64_t k = 0; k < group; ++k) {
        if (!std::isfinite(v[k])) return false;
        top = std::max(top, std::fabs(v[k]));
      }
      const uint16_t bits = bf16_bits(top / 7.f);
      const float s = bf16_value(bits);
      if (!std::isfinite(s)) return false;
      scales[n * (K / group) + g] = bits;
      for (int64_t k = 0; k < group; k += 2) {
        uint8_t c[2];
        for (int h = 0; h < 2; ++h) {
          // the scale is rounded, so the largest weight may lie just beyond 7 of it
          const float q = s > 0.f ? std::nearbyint(v[k + h] / s) : 0.f;
          c[h] = (uint8_t)((int)std::max(-7.f, std::min(7.f, q)) + 8);
        }
        codes[(n * K + g * group + k) / 2] = (uint8_t)(c[0] | c[1] << 4);
      }
    }
  return true;
}

}  // namespace tp

using namespace tp;

extern "C" {

tp_status tpo_w4_bytes(int32_t N, int32_t K, int32_t group, uint64_t* code_bytes, uint64_t* scale_bytes) {
  if (!code_bytes || !scale_bytes) return fail(TP_E_INVAL, "tpo_w4_bytes: NULL output");
  if (!w4_shape_ok(N, K, group))
    return fail(TP_E_INVAL, "tpo_w4_bytes: need 1 <= N <= 2^24, 1 <= K <= 2^20, group 32, 64 or 128 dividing K");
  *code_bytes = w4_code_bytes(N, K);
  *scale_bytes = w4_scale_bytes(N, K, group);
  return ok();
}

tp_status tpo_w4_pack(const uint8_t* codes, const uint16_t* scales, int32_t N, int32_t K, int32_t group,
                      uint8_t* codes_out, uint16_t* scales_out) {
  if (!codes || !scales || !codes_out || !scales_out) return fail(TP_E_INVAL, "tpo_w4_pack: NULL argument");
  if (!w4_shape_ok(N, K, group))
    return fail(TP_E_INVAL, "tpo_w4_pack: need 1 <= N <= 2^24, 1 <= K <= 2^20, group 32, 64 or 128 dividing K");
  w4_pack_codes(codes, N, K, codes_out);
  w4_pack_scales(scales, N, K, group, scales_out);
  return ok();
}

tp_status tpo_w4_quantize(const float* w, int32_t N, int32_t K, int32_t group, uint8_t* codes, uint16_t* scales) {
  if (!w || !codes || !scales) return fail(TP_E_INVAL, "tpo_w4_quantize: NULL argument");
  if (!w4_shape_ok(N, K, group))
    return fail(TP_E_INVAL, "tpo_w4_quantize: need 1 <= N <= 2^24, 1 <= K <= 2^20, group 32, 64 or 128 dividing K");
  if (!w4_quantize(w, N, K, group, codes, scales))
    return fail(TP_E_INVAL, "tpo_w4_quantize: a weight is not finite, or too large for a bf16 scale");
  return ok();
}

}  // extern "C"
