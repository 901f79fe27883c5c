// Packs and quantises matrices in buffers of exactly the sizes the 4-bit format asks for, so that AddressSanitizer sees any
// access beyond them, and checks that blocked scales and codes come back from their places.
#include <cmath>
#include <cstdint>
#include <cstdio>
#include <cstdlib>
#include <memory>

#include "torpor_ops.h"

static uint32_t state = 1;
static uint32_t rnd() { return state = state * 1664525u + 1013904223u; }

static int one(int n, int k, int group) {
  uint64_t cb = 0, sb = 0;
  if (tpo_w4_bytes(n, k, group, &cb, &sb) != TP_OK) return 1;
  const int64_t ng = k / group, kb = (k + 127) / 128;
  std::unique_ptr<float[]> w(new float[(size_t)n * k]);
  std::unique_ptr<uint8_t[]> codes(new uint8_t[(size_t)n * k / 2]), packed(new uint8_t[cb]);
  std::unique_ptr<uint16_t[]> scales(new uint16_t[n * ng]), pscales(new uint16_t[sb / 2]);
  for (int64_t i = 0; i < (int64_t)n * k; ++i) w[i] = ((int32_t)rnd() >> 8) * 1e-6f;
  if (tpo_w4_quantize(w.get(), n, k, group, codes.get(), scales.get()) != TP_OK) return 2;
  if (tpo_w4_pack(codes.get(), scales.get(), n, k, group, packed.get(), pscales.get()) != TP_OK) return 3;
  for (int64_t r = 0; r < n; ++r)
    for (int64_t c = 0; c < k; ++c) {
      const int64_t word = (r / 16 * kb + c / 128) * 256 + 4 * (16 * (c % 32 / 8) + r % 16) + c % 128 / 32;
      const int at = 4 * (int)(c % 8 / 2) + 16 * (int)(c % 2);
      uint32_t v = 0;
      for (int b = 0; b < 4; ++b) v |= (uint32_t)packed[word * 4 + b] << (8 * b);
      const uint32_t plain = codes[(r * k + c) / 2] >> (c % 2 ? 4 : 0) & 15;
      if ((v >> at & 15) != plain) return 4;
      if (pscales[(r / 16 * (kb * 128 / group) + c / group) * 16 + r % 16] != scales[r * ng + c / group]) return 5;
    }
  // too large for a bf16 scale, infinite, not a number: refused
  for (float odd : {3.4e38f, INFINITY, (float)NAN}) {
    w[(size_t)n * k - 1] = odd;
    const tp_status st = tpo_w4_quantize(w.get(), n, k, group, codes.get(), scales.get());
    if (std::isfinite(odd) ? st != TP_OK : st != TP_E_INVAL) return 6;
  }
  return 0;
}

int main() {
  for (int n : {1, 2, 15, 16, 17, 33, 100})
    for (int k : {32, 64, 96, 128, 160, 384, 1024})
      for (int group : {32, 64, 128}) {
        if (k % group) continue;
        if (int e = one(n, k, group)) {
          std::printf("%d x %d, groups of %d: check %d\n", n, k, group, e);
          return 1;
        }
      }
  uint64_t a, b;
  const int bad[][3] = {{0, 128, 128}, {1, 0, 32}, {1, 100, 32}, {1, 128, 16}, {-1, 128, 128}, {(1 << 24) + 1, 128, 128}, {1, (1 << 20) + 128, 128}};
  for (const auto& s : bad)
    if (tpo_w4_bytes(s[0], s[1], s[2], &a, &b) != TP_E_INVAL) return 1;
  return tpo_w4_bytes(1 << 24, 1 << 20, 32, &a, &b) == TP_OK && a == 1ull << 43 ? 0 : 1;
}
