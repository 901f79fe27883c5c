// Rows of keys and values into the pages of a cache and out of them (torpor_serve.h), on gfx950.
//
// A lane moves eight values, D / 8 lanes one token's head; rows are numbered sequence, row, k or v, head, so that
// lanes side by side read and write what lies side by side in the usual layouts. Each lane finds its page by itself: two lengths
// and a table entry, which the lanes of a token share in the caches.
//
// 8-bit rows: a = max |x| over the finite values of the head (a butterfly over its lanes), s = 2^e the smallest power of two
// with a <= 448 s = 1.75 2^8 s: for a = m 2^x, 1 <= m < 2, e = x - 8, or x - 7 where m > 1.75. Division by s is exact (a power of two), so
// the one rounding is the conversion's. Reading back, code * s has four significant bits: exact in bf16 unless it leaves its range.
#include "serve_args.hpp"

namespace tp {
namespace k {
namespace {

// Where lane `id` of a call works: sequence, row, k or v, head, chunk of eight values, page (negative: none) and token of it.
struct Place {
  int b, i, kv, h, ch, page, at;
  bool row;                         // a row that the sequence has
};

template <int CPH>
__device__ __forceinline__ Place place_of(const CacheRows& a, int id) {
  Place p;
  p.ch = id % CPH;
  int v = id / CPH;
  p.h = v % a.c.heads;
  v /= a.c.heads;
  p.kv = v & 1;
  v >>= 1;
  p.i = v % a.p.q_len;
  p.b = v / a.p.q_len;
  const Lens l = lens_of(a.p, p.b);
  p.row = p.i < l.qn;
  const int pos = l.kn - l.qn + p.i, col = pos >> a.c.lg;
  p.page = -1;
  if (p.row && pos >= 0 && col < a.p.max_pages) {
    const int page = a.p.table[(int64_t)p.b * a.p.table_stride + col];
    if ((unsigned)page < (unsigned)a.c.pages) p.page = page;
  }
  p.at = pos & ((1 << a.c.lg) - 1);
  return p;
}

__device__ __forceinline__ uint16_t* row_at(const CacheRows& a, const Place& p) {
  const int64_t* s = p.kv ? a.rvs : a.rks;
  return (p.kv ? a.v : a.k) + p.b * s[0] + p.i * s[1] + p.h * s[2] + 8 * p.ch;
}
template <bool E4M3>
__device__ __forceinline__ char* cell_at(const CacheRows& a, const Place& p) {
  const int64_t* s = p.kv ? a.c.vs : a.c.ks;
  return static_cast<char*>(p.kv ? a.c.v : a.c.k) + p.page * s[0] + p.at * s[1] + p.h * s[2] + (E4M3 ? 8 : 16) * p.ch;
}
__device__ __forceinline__ uint8_t* exp_at(const CacheRows& a, const Place& p) {
  return a.c.exps + ((((int64_t)p.page * 2 + p.kv) * a.c.heads + p.h) << a.c.lg) + p.at;
}

template <int D, bool E4M3>
__global__ __launch_bounds__(256) void k_cache_append(CacheRows a, int lanes) {
  constexpr int CPH = D / 8;
  const int id = blockIdx.x * 256 + threadIdx.x;
  const Place p = place_of<CPH>(a, min(id, lanes - 1));
  const bool live = id < lanes && p.page >= 0;      // the same for the lanes of a head
  if (!live) return;
  const uint4 w = *reinterpret_cast<const uint4*>(row_at(a, p));
  char* cell = cell_at<E4M3>(a, p);
  if constexpr (!E4M3) {
    *reinterpret_cast<uint4*>(cell) = w;
  } else {
    const uint32_t u[4] = {w.x, w.y, w.z, w.w};
    uint32_t top = 0;                               // bf16 bits of the largest finite magnitude
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const uint32_t lo = u[j] & 0x7fffu, hi = u[j] >> 16 & 0x7fffu;
      top = max(top, max(lo < 0x7f80u ? lo : 0u, hi < 0x7f80u ? hi : 0u));
    }
#pragma unroll
    for (int m = CPH / 2; m > 0; m >>= 1) top = max(top, (uint32_t)__shfl_xor((int)top, m, 64));
    // exponent bits of a, and one more where its seven mantissa bits are over those of 1.75
    const int byte = max((int)((top + 0x1fu) >> 7) - 8, 1);
    const float inv = __uint_as_float((uint32_t)(254 - byte) << 23);
    uint32_t c[2] = {0, 0};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const float lo = __uint_as_float(u[j] << 16) * inv, hi = __uint_as_float(u[j] & 0xffff0000u) * inv;
      const uint32_t pair = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(lo, hi, 0, false) & 0xffffu;
      c[j / 2] |= pair << (16 * (j & 1));
    }
    *reinterpret_cast<uint2*>(cell) = make_uint2(c[0], c[1]);
    if (p.ch == 0) *exp_at(a, p) = (uint8_t)byte;
  }
}

template <int D, bool E4M3>
__global__ __launch_bounds__(256) void k_cache_read(CacheRows a, int lanes) {
  constexpr int CPH = D / 8;
  const int id = blockIdx.x * 256 + threadIdx.x;
  if (id >= lanes) return;
  const Place p = place_of<CPH>(a, id);
  if (!p.row) return;
  uint4 w = make_uint4(0, 0, 0, 0);
  if (p.page >= 0) {
    const char* cell = cell_at<E4M3>(a, p);
    if constexpr (!E4M3) {
      w = *reinterpret_cast<const uint4*>(cell);
    } else {
      const uint2 c = *reinterpret_cast<const uint2*>(cell);
      const float s = __uint_as_float((uint32_t)*exp_at(a, p) << 23);
      auto two = [&](uint32_t x, auto high) {
        const bf16x2 v = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x, 1.f, decltype(high)::value);
        const uint32_t b = __builtin_bit_cast(uint32_t, v);
        return f2bf2(__uint_as_float(b << 16) * s, __uint_as_float(b & 0xffff0000u) * s);
      };
      w = make_uint4(two(c.x, std::false_type()), two(c.x, std::true_type()), two(c.y, std::false_type()), two(c.y, std::true_type()));
    }
  }
  *reinterpret_cast<uint4*>(row_at(a, p)) = w;
}

// Lanes of a call, or 0 for one that the kernels cannot take.
int lanes_of(const CacheRows& a) {
  if (!a.c.k || !a.c.v || (a.c.e4m3 && !a.c.exps) || !a.p.table || !a.p.kv_lens || !a.k || !a.v || (a.c.dim != 64 && a.c.dim != 128) ||
      a.p.batch < 1 || a.p.q_len < 1 || a.c.heads < 1 || a.c.pages < 1 || a.p.max_pages < 1 || a.c.lg < 4 || a.c.lg > 12)
    return 0;
  const int64_t heads = (int64_t)a.p.batch * a.p.q_len * a.c.heads;
  return heads < 1 << 26 ? (int)(heads * 2 * (a.c.dim / 8)) : 0;
}

template <typename F64, typename F128>
hipError_t go(const CacheRows& a, hipStream_t s, F64 k64, F128 k128) {
  const int lanes = lanes_of(a);
  if (!lanes) return hipErrorInvalidValue;
  return launch(a.c.dim == 64 ? k64 : k128, dim3(((unsigned)lanes + 255) / 256), dim3(256), 0, s, a, lanes);
}

}  // namespace

hipError_t cache_append(const CacheRows& a, hipStream_t s) {
  return a.c.e4m3 ? go(a, s, k_cache_append<64, true>, k_cache_append<128, true>) : go(a, s, k_cache_append<64, false>, k_cache_append<128, false>);
}

hipError_t cache_read(const CacheRows& a, hipStream_t s) {
  return a.c.e4m3 ? go(a, s, k_cache_read<64, true>, k_cache_read<128, true>) : go(a, s, k_cache_read<64, false>, k_cache_read<128, false>);
}

}  // namespace k
}  // namespace tp
