// Low-rank adapters of many requests beside a shared projection (torpor_serve.h): y[m] = act(base[m] + s_a B_a (A_a x[m])),
// a = adapter[m], on gfx950 MFMA (v_mfma_f32_16x16x32_bf16).
//
// A workgroup takes 16 rows and 256 outputs. It goes through the adapters that its rows name, one at a time, computes t = s A x for all
// 16 rows, and adds B t to those that have this adapter: a row's results are chosen, not multiplied by 0, so that no other
// row's values or adapter reach it. t is kept as two bf16 parts (high and rest: 2^-16 of t), both multiplied by B, so that
// fp32 results are fp32 results; the weights are bf16 as they are.
//
// Operands: first product A's rows r against x's rows m (t^T), the waves side by side along k, joined in LDS in wave
// order; second product B's rows n against t's rows m (y^T), rows of four blocks interleaved so that a lane ends with 16 consecutive
// outputs of its row. Rows of A behind the rank, and columns of B, are taken as zeros whatever they hold.
#include "serve_args.hpp"

namespace tp {
namespace k {
namespace {

constexpr int kMostRank = 128, kWaves = 4, kTileN = 64 * kWaves;

__device__ __forceinline__ uint4 zeros() { return make_uint4(0, 0, 0, 0); }

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

template <bool F32>
__global__ __launch_bounds__(64 * kWaves) void k_lora(Lora a, int tiles_n, bool vec) {
  __shared__ float part[kWaves][kMostRank][17];
  __shared__ __attribute__((aligned(16))) uint16_t th[16][kMostRank + 8], tl[16][kMostRank + 8];
  const int tid = threadIdx.x, lane = tid & 63, r16 = lane & 15, q4 = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int m0 = (int)(blockIdx.x / tiles_n) * 16, n0 = (int)(blockIdx.x % tiles_n) * kTileN + wave * 64;
  const int m = m0 + r16;
  const bool row = m < a.M;
  int mine = row ? a.adapter[m] : -1;
  if ((unsigned)mine >= (unsigned)a.adapters) mine = -1;
  const uint16_t* x = a.x + (int64_t)(row ? m : m0) * a.ldx;

  f32x4 acc[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) acc[e] = f32x4{0, 0, 0, 0};
  uint32_t left = (uint32_t)__ballot(mine >= 0) & 0xffffu;
  while (left) {
    const int ad = __builtin_amdgcn_readlane(mine, __builtin_ctz(left));
    const bool on = mine == ad;
    left &= ~(uint32_t)__ballot(on);
    const int rank = a.ranks ? min(max(a.ranks[ad], 0), a.R) : a.R;
    if (rank == 0) continue;
    const uint16_t* down = a.a + ad * a.as;
    const uint16_t* up = a.b + ad * a.bs;
    f32x4 d[kMostRank / 16];
#pragma unroll
    for (int rb = 0; rb < kMostRank / 16; ++rb) d[rb] = f32x4{0, 0, 0, 0};
    for (int k0 = wave * 32; k0 < a.K; k0 += 32 * kWaves) {
      const int k = k0 + 8 * q4;
      const bool in = k < a.K;                      // K is a multiple of 8
      const uint4 xf = in && row ? *reinterpret_cast<const uint4*>(x + k) : zeros();
#pragma unroll
      for (int rb = 0; rb < kMostRank / 16; ++rb) {
        if (rb * 16 >= rank) break;
        const int r = rb * 16 + r16;
        const uint4 af = in && r < rank ? *reinterpret_cast<const uint4*>(down + (int64_t)r * a.K + k) : zeros();
        d[rb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(af), as_bf16x8(xf), d[rb], 0, 0, 0);
      }
    }
    __syncthreads();                                // (the last adapter's t has been read)
#pragma unroll
    for (int rb = 0; rb < kMostRank / 16; ++rb) {
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
      const uint16_t hi = f2bf(t);
      const float rest = t - bf2f(hi);
      th[c][r] = hi;
      tl[c][r] = fabsf(t) < INFINITY ? f2bf(rest) : 0;
    }
    __syncthreads();
    f32x4 y[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) y[e] = f32x4{0, 0, 0, 0};
    for (int rc = 0; rc < rank; rc += 32) {
      const int r = rc + 8 * q4;
      const bf16x8 hf = as_bf16x8(*reinterpret_cast<const uint4*>(&th[r16][r]));
      const bf16x8 lf = as_bf16x8(*reinterpret_cast<const uint4*>(&tl[r16][r]));
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int n = n0 + 16 * (r16 >> 2) + 4 * e + (r16 & 3);
        const uint4 bf = n < a.N && r < rank ? first_of(*reinterpret_cast<const uint4*>(up + (int64_t)n * a.R + r), rank - r) : zeros();
        y[e] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(bf), hf, y[e], 0, 0, 0);
        y[e] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(bf), lf, y[e], 0, 0, 0);
      }
    }
    if (on) {
#pragma unroll
      for (int e = 0; e < 4; ++e) acc[e] = y[e];
    }
  }

  // lane holds outputs n0 + 16 q4 + 4 e + i of its row
  if (!row) return;
  const int n = n0 + 16 * q4;
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
        if (a.base) w = *reinterpret_cast<const uint4*>(bp + 4 * e);
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
    if (n + j >= a.N) break;
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

}  // namespace

hipError_t lora(const Lora& a, const Split& sp, hipStream_t s) {
  (void)sp;
  if (!a.x || !a.a || !a.b || !a.adapter || !a.y || a.M < 1 || a.N < 1 || a.K < 8 || a.K % 8 || a.R < 8 || a.R % 8 || a.R > kMostRank ||
      a.adapters < 1)
    return hipErrorInvalidValue;
  const int64_t tm = ((int64_t)a.M + 15) / 16, tn = ((int64_t)a.N + kTileN - 1) / kTileN;
  if (tm * tn >= 1 << 24) return hipErrorInvalidValue;
  const int64_t run = a.f32 ? 4 : 8;
  const bool vec = (uintptr_t)a.y % 16 == 0 && a.ldy % run == 0 && (uintptr_t)a.base % 16 == 0 && (!a.base || a.ldbase % run == 0);
  return launch(a.f32 ? k_lora<true> : k_lora<false>, dim3((unsigned)(tm * tn)), dim3(64 * kWaves), 0, s, a, (int)tn, vec);
}

}  // namespace k
}  // namespace tp
