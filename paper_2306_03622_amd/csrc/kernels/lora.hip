// Low-rank adapters of many requests beside a shared projection (torpor_serve.h): y[m] = act(base[m] + s_a B_a (A_a x[m])),
// a = adapter[m], on gfx950 MFMA (v_mfma_f32_16x16x32_bf16).
//
// Two launches: k_lora_down computes t = s A x (fp32, in `work`), k_lora_up adds B t to the base. In both a workgroup (or wave) takes a tile of
// rows, finds the adapters that they name (the rows' numbers lie one in a lane; a ballot gives an adapter's rows), and takes
// the rows of one adapter together, in blocks of 16, wherever in the tile they stand: rows of many requests in any order need no
// sorting, and no row meets another's adapter. Where there are few tiles, the adapters of a tile go to several workgroups.
// Without scratch k_lora does both in one launch and computes t anew for every 256 outputs.
//
// t is taken as bf16 parts (two, three for fp32 results: 2^-16 and 2^-24 of t), all multiplied by B, whose values are bf16 as they are.
// Operands: A's rows r against x's rows m (t^T), then B's rows n against t's rows m (y^T), rows n of four blocks interleaved so
// that a lane ends with 16 consecutive outputs of its row. What lies behind a rank is not used, whatever it holds.
#include "lora_plan.hpp"
#include "serve_args.hpp"

namespace tp {
namespace k {

struct LoraArgs {
  Lora a;
  float* t;               // [splits][M][R]
  int splits;             // over K
  int slots;              // workgroups (or waves) that share a tile's adapters
  int tiles_n;            // blocks of outputs
  int vec;                // base and y in whole 16 bytes
};

template <>
struct PtrFields<LoraArgs> {
  static void add(std::vector<uint32_t>& v, uint32_t at) {
    PtrFields<Lora>::add(v, at + (uint32_t)offsetof(LoraArgs, a));
    v.push_back(at + (uint32_t)offsetof(LoraArgs, t));
  }
};

namespace {

__device__ __forceinline__ uint4 zeros() { return make_uint4(0, 0, 0, 0); }
__device__ __forceinline__ uint4 load16(const void* p) { return *reinterpret_cast<const uint4*>(p); }

// bf16 pairs of a chunk of eight values, those from `n` on as zeros
__device__ __forceinline__ uint4 first_of(uint4 v, int n) {
  uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int j = 0; j < 4; ++j) w[j] &= n >= 2 * j + 2 ? 0xffffffffu : n == 2 * j + 1 ? 0xffffu : 0u;
  return make_uint4(w[0], w[1], w[2], w[3]);
}

__device__ __forceinline__ float lora_act(float v, int act) {
  if (act == ACT_RELU) return v < 0.f ? 0.f : v;      // keeps NaN
  return act_apply(v, act);
}

__device__ __forceinline__ int rank_of(const Lora& a, int ad) { return a.ranks ? min(max(a.ranks[ad], 0), a.R) : a.R; }

// The rest of t behind its bf16 part (none behind an infinity or NaN).
__device__ __forceinline__ float rest_of(float t, uint16_t part) { return fabsf(t) < INFINITY ? t - bf2f(part) : 0.f; }

// 16 outputs of row m from n on: base, activation, rounding.
template <bool F32>
__device__ __forceinline__ void finish(const Lora& a, bool vec, int m, int n, const f32x4 (&acc)[4]) {
  if (n >= a.N) return;
  if (vec && n + 16 <= a.N) {
    if constexpr (F32) {
      const float* bp = static_cast<const float*>(a.base) + m * a.ldbase + n;
      float* yp = static_cast<float*>(a.y) + m * a.ldy + n;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        f32x4 v = acc[e];
        if (a.base) v += *reinterpret_cast<const f32x4*>(bp + 4 * e);
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = lora_act(v[i], a.act);
        *reinterpret_cast<f32x4*>(yp + 4 * e) = v;
      }
    } else {
      const uint16_t* bp = static_cast<const uint16_t*>(a.base) + m * a.ldbase + n;
      uint16_t* yp = static_cast<uint16_t*>(a.y) + m * a.ldy + n;
#pragma unroll
      for (int e = 0; e < 4; e += 2) {
        uint4 w = zeros();
        if (a.base) w = load16(bp + 4 * e);
        uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float lo = lora_act(acc[e + j / 2][2 * (j % 2)] + __uint_as_float(u[j] << 16), a.act);
          const float hi = lora_act(acc[e + j / 2][2 * (j % 2) + 1] + __uint_as_float(u[j] & 0xffff0000u), a.act);
          u[j] = f2bf2(lo, hi);
        }
        *reinterpret_cast<uint4*>(yp + 4 * e) = make_uint4(u[0], u[1], u[2], u[3]);
      }
    }
    return;
  }
#pragma unroll
  for (int j = 0; j < 16; ++j) {
    if (n + j >= a.N) continue;
    float v = acc[j / 4][j % 4];
    if constexpr (F32) {
      if (a.base) v += static_cast<const float*>(a.base)[m * a.ldbase + n + j];
      static_cast<float*>(a.y)[m * a.ldy + n + j] = lora_act(v, a.act);
    } else {
      if (a.base) v += bf2f(static_cast<const uint16_t*>(a.base)[m * a.ldbase + n + j]);
      static_cast<uint16_t*>(a.y)[m * a.ldy + n + j] = f2bf(lora_act(v, a.act));
    }
  }
}

// The adapter of row m0 + lane (lanes below ROWS), -1: none.
template <int ROWS>
__device__ __forceinline__ int adapter_at(const Lora& a, int m0, int lane) {
  const int id = lane < ROWS && m0 + lane < a.M ? a.adapter[m0 + lane] : -1;
  return (unsigned)id < (unsigned)a.adapters ? id : -1;
}

// Lane j holds the number of the j-th set bit of `mask` (behind the last: 0).
__device__ __forceinline__ int nth_of(unsigned long long mask, int lane) {
  const int before = (int)__builtin_amdgcn_mbcnt_hi((uint32_t)(mask >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)mask, 0));
  // lanes without a bit send to lane 63, where the last bit's lane sends too if all 64 are set: then no lane is without
  return __builtin_amdgcn_ds_permute((mask >> lane & 1 ? before : 63) * 4, mask >> lane & 1 ? lane : 0);
}

// t[z][m][r] of the rows of 32 that name an adapter of this slot: the waves side by side along k in steps of 32, joined in LDS in
// wave order. RB: blocks of 16 ranks.
template <int RB, int W>
__global__ __launch_bounds__(64 * W) void k_lora_down(LoraArgs g) {
  __shared__ float part[W][16][33];
  const Lora& a = g.a;
  const int tid = threadIdx.x, lane = tid & 63, r16 = lane & 15, q4 = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  int at = blockIdx.x;
  const int z = at % g.splits;
  at /= g.splits;
  const int slot = at % g.slots, m0 = at / g.slots * 32;
  const int mine = adapter_at<32>(a, m0, lane);
  const int full = a.K >> 5, stride = g.splits * W;

  auto body = [&](auto blocks, int ad, int rows, int count) __attribute__((always_inline)) {
    constexpr int MB = decltype(blocks)::value;
    const int rank = rank_of(a, ad);
    int m[MB];
    const uint16_t *x[MB], *down[RB];
#pragma unroll
    for (int mb = 0; mb < MB; ++mb) {
      const int j = mb * 16 + r16;
      m[mb] = m0 + __shfl(rows, j < count ? j : 0, 64);         // behind the last: the first again, not written
      x[mb] = a.x + m[mb] * a.ldx + 8 * q4;
    }
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) down[rb] = a.a + ad * a.as + (int64_t)min(rb * 16 + r16, a.R - 1) * a.K + 8 * q4;
    f32x4 d[RB][MB];
#pragma unroll
    for (int rb = 0; rb < RB; ++rb)
#pragma unroll
      for (int mb = 0; mb < MB; ++mb) d[rb][mb] = f32x4{0, 0, 0, 0};
    auto multiply = [&](const uint4 (&xf)[MB], const uint4 (&af)[RB]) __attribute__((always_inline)) {
#pragma unroll
      for (int rb = 0; rb < RB; ++rb)
#pragma unroll
        for (int mb = 0; mb < MB; ++mb)
          d[rb][mb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(af[rb]), as_bf16x8(xf[mb]), d[rb][mb], 0, 0, 0);
    };
    int s = z * W + wave;
    constexpr int U = RB > 4 ? 2 : 4;               // steps loaded together
    for (; s + (U - 1) * stride < full; s += U * stride) {
      uint4 xf[U][MB], af[U][RB];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int k = (s + u * stride) * 32;
#pragma unroll
        for (int mb = 0; mb < MB; ++mb) xf[u][mb] = load16(x[mb] + k);
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) af[u][rb] = load16(down[rb] + k);
      }
#pragma unroll
      for (int u = 0; u < U; ++u) multiply(xf[u], af[u]);
    }
    for (; s * 32 < a.K; s += stride) {
      const int k = s * 32;
      const bool in = k + 8 * q4 < a.K;             // K is a multiple of 8
      uint4 xf[MB], af[RB];
#pragma unroll
      for (int mb = 0; mb < MB; ++mb) xf[mb] = in ? load16(x[mb] + k) : zeros();
#pragma unroll
      for (int rb = 0; rb < RB; ++rb) af[rb] = in ? load16(down[rb] + k) : zeros();
      multiply(xf, af);
    }
    const float scale = a.scales ? a.scales[ad] : 1.f;
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
      __syncthreads();                              // (what was there has been read)
#pragma unroll
      for (int mb = 0; mb < MB; ++mb)
#pragma unroll
        for (int i = 0; i < 4; ++i) part[wave][4 * q4 + i][mb * 16 + r16] = d[rb][mb][i];
      __syncthreads();
      for (int i = tid; i < 16 * 16 * MB; i += 64 * W) {
        const int r = rb * 16 + i % 16, j = i / 16;
        float t = 0.f;
#pragma unroll
        for (int w = 0; w < W; ++w) t += part[w][i % 16][j];
        const int row = __shfl(rows, min(j, 31), 64);
        if (j < count && r < a.R) g.t[((int64_t)z * a.M + m0 + row) * a.R + r] = r < rank ? t * scale : 0.f;
      }
    }
  };
  unsigned long long left = __ballot(mine >= 0);
  for (int j = 0; left; ++j) {
    const int ad = __builtin_amdgcn_readlane(mine, (int)__builtin_ctzll(left));
    const unsigned long long mask = __ballot(mine == ad);
    left &= ~mask;
    if (j % g.slots != slot) continue;
    const int rows = nth_of(mask, lane), count = __builtin_popcountll(mask);
    if (count > 16) body(std::integral_constant<int, 2>(), ad, rows, count);
    else body(std::integral_constant<int, 1>(), ad, rows, count);
  }
}

// y of the rows of 64 that name an adapter of this slot (slot 0: those without one too), 64 outputs a wave. RC: chunks of 32 ranks.
template <bool F32, int RC>
__global__ __launch_bounds__(256) void k_lora_up(LoraArgs g) {
  constexpr int PARTS = F32 ? 3 : 2;
  const Lora& a = g.a;
  const int lane = threadIdx.x & 63, r16 = lane & 15, q4 = lane >> 4;
  int at = blockIdx.x;
  const int n0 = (at % g.tiles_n * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6)) * 64;
  at /= g.tiles_n;
  const int slot = at % g.slots, m0 = at / g.slots * 64;
  if (n0 >= a.N) return;
  const int mine = adapter_at<64>(a, m0, lane);

  auto body = [&](auto blocks, int ad, int rows, int first, int count) __attribute__((always_inline)) {
    constexpr int MB = decltype(blocks)::value;
    int m[MB];
#pragma unroll
    for (int mb = 0; mb < MB; ++mb) {
      const int j = first + mb * 16 + r16;
      m[mb] = m0 + __shfl(rows, j < count ? j : 0, 64);
    }
    f32x4 acc[MB][4];
#pragma unroll
    for (int mb = 0; mb < MB; ++mb)
#pragma unroll
      for (int e = 0; e < 4; ++e) acc[mb][e] = f32x4{0, 0, 0, 0};
    const int rank = ad < 0 ? 0 : rank_of(a, ad);
    const uint16_t* up = a.b + max(ad, 0) * a.bs;
#pragma unroll
    for (int rc = 0; rc < RC; ++rc) {
      if (rc * 32 >= rank) break;
      const int r = rc * 32 + 8 * q4;
      const bool in = r < rank;
      uint4 bf[4], tf[MB][PARTS];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int n = min(n0 + 16 * (r16 >> 2) + 4 * e + (r16 & 3), a.N - 1);           // behind the last: not stored
        bf[e] = in ? load16(up + (int64_t)n * a.R + r) : zeros();
      }
#pragma unroll
      for (int mb = 0; mb < MB; ++mb) {
        float t[8] = {};
        if (in) {
          for (int z = 0; z < g.splits; ++z) {
            const float* p = g.t + ((int64_t)z * a.M + m[mb]) * a.R + r;
            const f32x4 lo = *reinterpret_cast<const f32x4*>(p), hi = *reinterpret_cast<const f32x4*>(p + 4);
#pragma unroll
            for (int i = 0; i < 4; ++i) t[i] += lo[i], t[4 + i] += hi[i];
          }
        }
#pragma unroll
        for (int p = 0; p < PARTS; ++p) {
          uint32_t w[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            w[i] = f2bf2(t[2 * i], t[2 * i + 1]);
            t[2 * i] = rest_of(t[2 * i], (uint16_t)w[i]);
            t[2 * i + 1] = rest_of(t[2 * i + 1], (uint16_t)(w[i] >> 16));
          }
          tf[mb][p] = make_uint4(w[0], w[1], w[2], w[3]);
        }
      }
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const bf16x8 b = as_bf16x8(first_of(bf[e], rank - r));
#pragma unroll
        for (int mb = 0; mb < MB; ++mb)
#pragma unroll
          for (int p = 0; p < PARTS; ++p) acc[mb][e] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(b, as_bf16x8(tf[mb][p]), acc[mb][e], 0, 0, 0);
      }
    }
    // lane holds outputs n0 + 16 q4 + 4 e + i of its rows
#pragma unroll
    for (int mb = 0; mb < MB; ++mb)
      if (first + mb * 16 + r16 < count) finish<F32>(a, g.vec, m[mb], n0 + 16 * q4, acc[mb]);
  };
  auto rows_of = [&](unsigned long long mask, int ad) __attribute__((always_inline)) {
    const int rows = nth_of(mask, lane), count = __builtin_popcountll(mask);
    if (count > 32) {
      body(std::integral_constant<int, 4>(), ad, rows, 0, count);
    } else {
      for (int first = 0; first < count; first += 16) body(std::integral_constant<int, 1>(), ad, rows, first, count);
    }
  };
  unsigned long long left = __ballot(mine >= 0);
  const unsigned long long none = __ballot(m0 + lane < a.M) & ~left;
  if (slot == 0 && none) rows_of(none, -1);
  for (int j = 0; left; ++j) {
    const int ad = __builtin_amdgcn_readlane(mine, (int)__builtin_ctzll(left));
    const unsigned long long mask = __ballot(mine == ad);
    left &= ~mask;
    if (j % g.slots == slot) rows_of(mask, ad);
  }
}

// Both products in one launch, for 16 rows and 256 outputs; every adapter's results are chosen for its rows.
constexpr int kWaves = 4;

template <bool F32>
__global__ __launch_bounds__(64 * kWaves) void k_lora(LoraArgs g) {
  constexpr int PARTS = F32 ? 3 : 2;
  __shared__ float part[kWaves][kLoraRank][17];
  __shared__ __attribute__((aligned(16))) uint16_t ts[PARTS][16][kLoraRank + 8];
  const Lora& a = g.a;
  const int tid = threadIdx.x, lane = tid & 63, r16 = lane & 15, q4 = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int m0 = (int)(blockIdx.x / g.tiles_n) * 16, n0 = ((int)(blockIdx.x % g.tiles_n) * kWaves + wave) * 64;
  const int m = m0 + r16;
  const bool row = m < a.M;
  const int mine = __shfl(adapter_at<16>(a, m0, lane), r16, 64);
  const uint16_t* x = a.x + (row ? m : m0) * a.ldx;

  f32x4 acc[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) acc[e] = f32x4{0, 0, 0, 0};
  uint32_t left = (uint32_t)__ballot(mine >= 0) & 0xffffu;
  while (left) {
    const int ad = __builtin_amdgcn_readlane(mine, __builtin_ctz(left));
    const bool on = mine == ad;
    left &= ~(uint32_t)__ballot(on);
    const int rank = rank_of(a, ad);
    if (rank == 0) continue;
    const uint16_t* down = a.a + ad * a.as;
    const uint16_t* up = a.b + ad * a.bs;
    f32x4 d[kLoraRank / 16];
#pragma unroll
    for (int rb = 0; rb < kLoraRank / 16; ++rb) d[rb] = f32x4{0, 0, 0, 0};
    for (int k0 = wave * 32; k0 < a.K; k0 += 32 * kWaves) {
      const int k = k0 + 8 * q4;
      const bool in = k < a.K;                      // K is a multiple of 8
      const uint4 xf = in && row ? load16(x + k) : zeros();
#pragma unroll
      for (int rb = 0; rb < kLoraRank / 16; ++rb) {
        if (rb * 16 >= rank) break;
        const int r = rb * 16 + r16;
        const uint4 af = in && r < rank ? load16(down + (int64_t)r * a.K + k) : zeros();
        d[rb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(af), as_bf16x8(xf), d[rb], 0, 0, 0);
      }
    }
    __syncthreads();                                // (the last adapter's t has been read)
#pragma unroll
    for (int rb = 0; rb < kLoraRank / 16; ++rb) {
      if (rb * 16 >= rank) break;
#pragma unroll
      for (int i = 0; i < 4; ++i) part[wave][rb * 16 + 4 * q4 + i][r16] = d[rb][i];
    }
    __syncthreads();
    const float scale = a.scales ? a.scales[ad] : 1.f;
    for (int i = tid; i < (rank + 31) / 32 * 32 * 16; i += 64 * kWaves) {
      const int r = i >> 4, c = i & 15;
      float t = 0.f;
      if (r < rank) {
#pragma unroll
        for (int w = 0; w < kWaves; ++w) t += part[w][r][c];
        t *= scale;
      }
#pragma unroll
      for (int p = 0; p < PARTS; ++p) {
        ts[p][c][r] = f2bf(t);
        t = rest_of(t, ts[p][c][r]);
      }
    }
    __syncthreads();
    f32x4 y[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) y[e] = f32x4{0, 0, 0, 0};
    for (int rc = 0; rc < rank; rc += 32) {
      const int r = rc + 8 * q4;
      bf16x8 tf[PARTS];
#pragma unroll
      for (int p = 0; p < PARTS; ++p) tf[p] = as_bf16x8(load16(&ts[p][r16][r]));
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int n = n0 + 16 * (r16 >> 2) + 4 * e + (r16 & 3);
        const uint4 bf = n < a.N && r < rank ? first_of(load16(up + (int64_t)n * a.R + r), rank - r) : zeros();
#pragma unroll
        for (int p = 0; p < PARTS; ++p) y[e] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(bf), tf[p], y[e], 0, 0, 0);
      }
    }
    if (on) {
#pragma unroll
      for (int e = 0; e < 4; ++e) acc[e] = y[e];
    }
  }
  // lane holds outputs n0 + 16 q4 + 4 e + i of its row
  if (row) finish<F32>(a, g.vec, m, n0 + 16 * q4, acc);
}

template <bool F32>
hipError_t up(const LoraArgs& g, unsigned wgs, hipStream_t s) {
  const int rc = (g.a.R + 31) / 32;
  return launch(rc == 1 ? k_lora_up<F32, 1> : rc == 2 ? k_lora_up<F32, 2> : k_lora_up<F32, 4>, dim3(wgs), dim3(256), 0, s, g);
}

}  // namespace

hipError_t lora(const Lora& a, const Split& sp, hipStream_t s) {
  if (!a.x || !a.a || !a.b || !a.adapter || !a.y || a.M < 1 || a.N < 1 || a.K < 8 || a.K % 8 || a.R < 8 || a.R % 8 || a.R > kLoraRank ||
      a.adapters < 1)
    return hipErrorInvalidValue;
  LoraArgs g{};
  g.a = a;
  g.t = sp.partials;
  g.tiles_n = (int)(((int64_t)a.N + 255) / 256);
  const int64_t run = a.f32 ? 4 : 8;
  g.vec = (uintptr_t)a.y % 16 == 0 && a.ldy % run == 0 && (uintptr_t)a.base % 16 == 0 && (!a.base || a.ldbase % run == 0);
  if (((int64_t)a.M + 15) / 16 * g.tiles_n >= 1 << 24) return hipErrorInvalidValue;
  const LoraPlan p = lora_plan(a.M, a.N, a.K, a.R, a.adapters, sp.partials ? sp.partial_bytes : 0);
  if (p.splits == 0)
    return launch(a.f32 ? k_lora<true> : k_lora<false>, dim3((unsigned)((a.M + 15) / 16 * g.tiles_n)), dim3(64 * kWaves), 0, s, g);
  g.splits = p.splits;
  g.slots = p.down_slots;
  const unsigned tiles = (a.M + 31) / 32;
  const int rb = (a.R + 15) / 16;
  const hipError_t e = launch(rb == 1 ? k_lora_down<1, 8> : rb == 2 ? k_lora_down<2, 8> : rb <= 4 ? k_lora_down<4, 8> : k_lora_down<8, 8>,
                              dim3(tiles * g.slots * g.splits), dim3(512), 0, s, g);
  if (e != hipSuccess) return e;
  g.slots = p.up_slots;
  const unsigned wgs = (unsigned)((a.M + 63) / 64) * g.slots * g.tiles_n;
  return a.f32 ? up<true>(g, wgs, s) : up<false>(g, wgs, s);
}

}  // namespace k
}  // namespace tp
