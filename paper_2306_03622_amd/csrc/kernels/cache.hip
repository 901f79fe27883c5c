// Rows of keys and values into the pages of a cache and out of them (torpor_serve.h), on gfx950.
//
// A lane moves eight values of a key and of its value, D / 8 lanes one token's head, lanes side by side what lies side by side in the
// usual layouts. A workgroup belongs to one sequence and takes U rows in each place, all of whose pages and then values are asked for
// before the first is waited for. What is left of the index arithmetic is scalar or once a lane (by divisions in every lane, reading 8191
// tokens of 8 heads of 128 in 8 bits took 14.8 us, now 10.5).
//
// 8-bit rows: a = max |x| over the finite values of the head, s = 2^e the smallest power of two
// with a <= 448 s = 1.75 2^8 s: for a = m 2^x, 1 <= m < 2, e = x - 8, or x - 7 where m > 1.75. Division by s is exact (a power of two), so
// the one rounding is the conversion's. Reading back, code * s has four significant bits: exact in bf16 unless it leaves its range.
#include "cache_plan.hpp"
#include "serve_args.hpp"

namespace tp {
namespace k {

struct CacheRowsArgs {
  CacheRows a;
  int per, cols, rows, blocks;      // CacheRowsPlan
};

namespace {

template <int CTRL>
__device__ __forceinline__ uint32_t dpp_max(uint32_t v) {
  return max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xF, 0xF, false));
}

// Eight values of a head in 8 bits: the head's exponent byte, the codes.
template <int CPH>
__device__ __forceinline__ uint2 to_e4m3(uint4 w, int* byte) {
  const uint32_t u[4] = {w.x, w.y, w.z, w.w};
  uint32_t top = 0;                                 // bf16 bits of the largest finite magnitude
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const uint32_t lo = u[j] & 0x7fffu, hi = u[j] >> 16 & 0x7fffu;
    top = max(top, max(lo < 0x7f80u ? lo : 0u, hi < 0x7f80u ? hi : 0u));
  }
  // over the head's lanes, all of which are there: mirrored in 16 and in 8 lanes, then inside four
  if constexpr (CPH == 16) top = dpp_max<0x140>(top);
  top = dpp_max<0x141>(top);
  top = dpp_max<0x4E>(top);
  top = dpp_max<0xB1>(top);
  // exponent bits of a, and one more where its seven mantissa bits are over those of 1.75
  *byte = max((int)((top + 0x1fu) >> 7) - 8, 1);
  const float inv = __uint_as_float((uint32_t)(254 - *byte) << 23);
  uint32_t c[2];
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    const int lo = __builtin_amdgcn_cvt_pk_fp8_f32(__uint_as_float(u[2 * j] << 16) * inv, __uint_as_float(u[2 * j] & 0xffff0000u) * inv, 0, false);
    c[j] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(__uint_as_float(u[2 * j + 1] << 16) * inv, __uint_as_float(u[2 * j + 1] & 0xffff0000u) * inv, lo, true);
  }
  return make_uint2(c[0], c[1]);
}

// Eight codes times 2^(byte - 127). The conversion takes its scale as an exponent byte, at an fp32 number's place of it: 0 is 2^-127
// there and 255 NaN (as a number to multiply by they are 0 and infinity), and its one rounding is to the nearest, ties to even.
__device__ __forceinline__ uint4 from_e4m3(uint2 c, uint32_t byte) {
  const float s = __uint_as_float(byte << 23);
  auto two = [&](uint32_t x, auto high) { return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x, s, decltype(high)::value)); };
  return make_uint4(two(c.x, std::false_type()), two(c.x, std::true_type()), two(c.y, std::false_type()), two(c.y, std::true_type()));
}

template <int D, bool E4M3, bool APPEND, int U>
__global__ __launch_bounds__(256) void k_cache_rows(CacheRowsArgs g) {
  constexpr int CPH = D / 8, CELL = E4M3 ? 8 : 16;
  const CacheRows& a = g.a;
  const Cache& c = a.c;
  int id = blockIdx.x;
  const int col = id % g.cols;
  id /= g.cols;
  const int block = id % g.blocks, b = id / g.blocks;
  const int sub = g.rows > 1 ? (int)threadIdx.x / g.per : 0, lane = (int)threadIdx.x - sub * g.per + col * 256;
  if (sub >= g.rows || lane >= g.per) return;       // whole heads
  const int h = lane / CPH, ch = lane % CPH;
  const Lens l = lens_of(a.p, b);
  const int32_t* table = a.p.table + b * a.p.table_stride;
  uint16_t* const rows[2] = {a.k + b * a.rks[0] + h * a.rks[2] + 8 * ch, a.v + b * a.rvs[0] + h * a.rvs[2] + 8 * ch};
  char* const cells[2] = {static_cast<char*>(c.k) + h * c.ks[2] + CELL * ch, static_cast<char*>(c.v) + h * c.vs[2] + CELL * ch};

  int row[U], page[U], at[U];
  auto row_at = [&](int n, int u) { return reinterpret_cast<uint4*>(rows[n] + row[u] * (n ? a.rvs[1] : a.rks[1])); };
  uint4 w[2][U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    row[u] = (block * U + u) * g.rows + sub;
#pragma unroll
    for (int n = 0; n < 2; ++n) w[n][u] = APPEND && row[u] < l.qn ? *row_at(n, u) : make_uint4(0, 0, 0, 0);
    const int pos = l.kn - l.qn + row[u], k = pos >> c.lg;
    page[u] = -1;
    at[u] = pos & ((1 << c.lg) - 1);
    if (row[u] < l.qn && pos >= 0 && k < a.p.max_pages) page[u] = table[k];
    if ((unsigned)page[u] >= (unsigned)c.pages) page[u] = -1;
  }
  auto cell_at = [&](int n, int u) { return cells[n] + page[u] * (n ? c.vs[0] : c.ks[0]) + at[u] * (n ? c.vs[1] : c.ks[1]); };
  auto exp_at = [&](int n, int u) { return c.exps + ((((int64_t)page[u] * 2 + n) * c.heads + h) << c.lg) + at[u]; };
  if constexpr (APPEND) {
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int n = 0; n < 2; ++n) {
        if (page[u] < 0) continue;                  // the same for the lanes of a head
        if constexpr (E4M3) {
          int byte;
          *reinterpret_cast<uint2*>(cell_at(n, u)) = to_e4m3<CPH>(w[n][u], &byte);
          if (ch == 0) *exp_at(n, u) = (uint8_t)byte;
        } else {
          *reinterpret_cast<uint4*>(cell_at(n, u)) = w[n][u];
        }
      }
  } else {
    uint32_t byte[2][U];
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int n = 0; n < 2; ++n) {
        byte[n][u] = 0;
        if (page[u] < 0) continue;
        if constexpr (E4M3) {
          const uint2 x = *reinterpret_cast<const uint2*>(cell_at(n, u));
          w[n][u].x = x.x, w[n][u].y = x.y;
          byte[n][u] = *exp_at(n, u);
        } else {
          w[n][u] = *reinterpret_cast<const uint4*>(cell_at(n, u));
        }
      }
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int n = 0; n < 2; ++n)
        if (row[u] < l.qn) *row_at(n, u) = E4M3 && page[u] >= 0 ? from_e4m3(make_uint2(w[n][u].x, w[n][u].y), byte[n][u]) : w[n][u];
  }
}

template <int D, bool E4M3, bool APPEND>
hipError_t go(CacheRowsArgs g, int64_t wgs, int u, hipStream_t s) {
  return launch(u == 1 ? k_cache_rows<D, E4M3, APPEND, 1> : k_cache_rows<D, E4M3, APPEND, 2>, dim3((unsigned)wgs), dim3(256), 0, s, g);
}

template <bool APPEND>
hipError_t rows(const CacheRows& a, hipStream_t s) {
  if (!a.c.k || !a.c.v || (a.c.e4m3 && !a.c.exps) || !a.p.table || !a.p.kv_lens || !a.k || !a.v || (a.c.dim != 64 && a.c.dim != 128) ||
      a.p.batch < 1 || a.p.q_len < 1 || a.c.heads < 1 || a.c.heads > 65536 || a.c.pages < 1 || a.p.max_pages < 1 || a.c.lg < 4 || a.c.lg > 12)
    return hipErrorInvalidValue;
  const CacheRowsPlan p = cache_rows_plan(a.c.dim, a.c.heads, a.p.batch, a.p.q_len);
  const int64_t wgs = p.blocks * p.cols * a.p.batch;
  if (wgs >= 1 << 24) return hipErrorInvalidValue;
  CacheRowsArgs g{};
  g.a = a;
  g.per = p.per, g.cols = p.cols, g.rows = p.rows, g.blocks = (int)p.blocks;
  if (a.c.e4m3) return a.c.dim == 64 ? go<64, true, APPEND>(g, wgs, p.each, s) : go<128, true, APPEND>(g, wgs, p.each, s);
  return a.c.dim == 64 ? go<64, false, APPEND>(g, wgs, p.each, s) : go<128, false, APPEND>(g, wgs, p.each, s);
}

}  // namespace

hipError_t cache_append(const CacheRows& a, hipStream_t s) { return rows<true>(a, s); }
hipError_t cache_read(const CacheRows& a, hipStream_t s) { return rows<false>(a, s); }

}  // namespace k
}  // namespace tp
