// Linear layers with 4-bit weights and a bf16 scale per group of columns (blocked order, torpor_ops.h) on gfx950
// MFMA: y[m][n] = act(sum_g s[n][g] sum_{k in g} (c[n][k] - 8) x[m][k] + bias[n] + res[m][n]).
//
// A code becomes a bf16 value in two instructions for a pair: shifted into the mantissa of 16.0 (0x4180, whose
// steps are 1/8: bits 3..6), the bits read 16 + c, exactly. The surplus of 24 on every weight is taken off by the sum
// of the activations: each group's accumulator starts from -24 sum_k x[m][k], which the matrix cores
// compute too, as a product with a constant operand. So every product is exact, the sums are fp32, and the scale
// multiplies a group's finished sum, in fp32: nothing is rounded to bf16 before the result. The surplus costs the
// sums about two bits: partial sums of 16 + c reach 31 |x| where the result's terms reach 8 |x|.
//
// Operand convention of the other contractions: A operand 16 weight rows, B operand 16 activation
// rows, accumulator register e of lane l holds D[n = 4 (l / 16) + e][m = l % 16].
#include "common.hpp"
#include "kernels.hpp"

namespace tp {
namespace k {

struct W4Args {
  LinearW4 a;
  int kb, groups;         // 128-column blocks, groups with padding
  int vec;                // outputs, bias and residual may be accessed as vectors of 4
};

template <>
struct PtrFields<W4Args> {
  static void add(std::vector<uint32_t>& v, uint32_t at) {
    for (size_t o : {offsetof(LinearW4, x), offsetof(LinearW4, wq), offsetof(LinearW4, scales), offsetof(LinearW4, bias),
                     offsetof(LinearW4, res), offsetof(LinearW4, y)})
      v.push_back(at + (uint32_t)(offsetof(W4Args, a) + o));
  }
};

namespace {

// eight codes as bf16 16 + c, column order
__device__ __forceinline__ bf16x8 w4_values(uint32_t w) {
  constexpr uint32_t mask = 0x00780078u, one = 0x41804180u;
  return as_bf16x8(make_uint4(((w << 3) & mask) | one, ((w >> 1) & mask) | one, ((w >> 5) & mask) | one,
                              ((w >> 9) & mask) | one));
}

// the constant operand -24 in every place
__device__ __forceinline__ bf16x8 w4_surplus() {
  return as_bf16x8(make_uint4(0xC1C0C1C0u, 0xC1C0C1C0u, 0xC1C0C1C0u, 0xC1C0C1C0u));
}

// outputs n0 .. n0 + 3 of row m
__device__ __forceinline__ void w4_store(const W4Args& g, int m, int n0, f32x4 acc) {
  const LinearW4& a = g.a;
  if (m >= a.M || n0 >= a.N) return;
  const int64_t at = (int64_t)m * a.ldy + n0;
  float v[4] = {acc[0], acc[1], acc[2], acc[3]};
  if (g.vec && n0 + 3 < a.N) {
    if (a.bias) {
      const uint2 w = *reinterpret_cast<const uint2*>(a.bias + n0);
      v[0] += bf2f(w.x & 0xffff); v[1] += bf2f(w.x >> 16); v[2] += bf2f(w.y & 0xffff); v[3] += bf2f(w.y >> 16);
    }
    if (a.res) {
      const uint2 w = *reinterpret_cast<const uint2*>(a.res + (int64_t)m * a.ldr + n0);
      v[0] += bf2f(w.x & 0xffff); v[1] += bf2f(w.x >> 16); v[2] += bf2f(w.y & 0xffff); v[3] += bf2f(w.y >> 16);
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = act_apply(v[e], a.act);
    if (a.y_f32) *reinterpret_cast<float4*>(static_cast<float*>(a.y) + at) = make_float4(v[0], v[1], v[2], v[3]);
    else *reinterpret_cast<uint2*>(static_cast<uint16_t*>(a.y) + at) = make_uint2(f2bf2(v[0], v[1]), f2bf2(v[2], v[3]));
    return;
  }
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    if (n0 + e >= a.N) break;
    float t = v[e];
    if (a.bias) t += bf2f(a.bias[n0 + e]);
    if (a.res) t += bf2f(a.res[(int64_t)m * a.ldr + n0 + e]);
    t = act_apply(t, a.act);
    if (a.y_f32) static_cast<float*>(a.y)[at + e] = t;
    else static_cast<uint16_t*>(a.y)[at + e] = f2bf(t);
  }
}

// Few rows: a workgroup owns 16 NB weight rows and 16 MT activation rows, its NW waves a contiguous run of k-blocks
// each; they add up through LDS in wave order. One 16-byte load per lane brings a whole 1 KB block.
template <int MT, int NB, int NW, int GP, int U>
__global__ __launch_bounds__(NW * 64) void k_w4_rows(W4Args g) {
  constexpr int SPG = 4 / GP;             // 32-column steps per group
  const LinearW4& a = g.a;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int r = lane & 15, q = lane >> 4;
  const int nb0 = blockIdx.x * NB, m0 = blockIdx.y * (16 * MT);
  const int nbs = (a.N + 15) >> 4;
  const uint16_t* xrow[MT];
  bool mvalid[MT];
#pragma unroll
  for (int t = 0; t < MT; ++t) {
    const int m = m0 + 16 * t + r;
    mvalid[t] = m < a.M;
    xrow[t] = a.x + (int64_t)(mvalid[t] ? m : 0) * a.ldx + (q << 3);
  }
  // a block row beyond the last reads the last one again; its outputs are not stored
  const uint8_t* wrow[NB];
  const uint16_t* srow[NB];
#pragma unroll
  for (int b = 0; b < NB; ++b) {
    const int nb = min(nb0 + b, nbs - 1);
    wrow[b] = a.wq + (int64_t)nb * g.kb * 1024 + lane * 16;
    srow[b] = a.scales + (int64_t)nb * g.groups * 16 + (q << 2);
  }
  f32x4 acc[NB][MT];
#pragma unroll
  for (int b = 0; b < NB; ++b)
#pragma unroll
    for (int t = 0; t < MT; ++t) acc[b][t] = f32x4{0.f, 0.f, 0.f, 0.f};
  const bf16x8 surplus = w4_surplus();
  const int per = (g.kb + NW - 1) / NW, kb_end = min(g.kb, (wave + 1) * per);
  for (int kb0 = wave * per; kb0 < kb_end; kb0 += U) {
    uint4 wv[U][NB], xv[U][MT][4];
    uint2 sv[U][NB][GP];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int kb = min(kb0 + u, kb_end - 1);
#pragma unroll
      for (int b = 0; b < NB; ++b) {
        wv[u][b] = load_nt16(wrow[b] + (int64_t)kb * 1024);
#pragma unroll
        for (int p = 0; p < GP; ++p) sv[u][b][p] = *reinterpret_cast<const uint2*>(srow[b] + (kb * GP + p) * 16);
      }
#pragma unroll
      for (int t = 0; t < MT; ++t)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int k0 = kb * 128 + 32 * j;
          uint4 v = make_uint4(0, 0, 0, 0);
          if (mvalid[t] && k0 < a.K) v = *reinterpret_cast<const uint4*>(xrow[t] + k0);
          xv[u][t][j] = v;
        }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (kb0 + u >= kb_end) break;
#pragma unroll
      for (int p = 0; p < GP; ++p) {
        f32x4 xs[MT];
#pragma unroll
        for (int t = 0; t < MT; ++t) {
          xs[t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int j = p * SPG; j < (p + 1) * SPG; ++j)
            xs[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(surplus, as_bf16x8(xv[u][t][j]), xs[t], 0, 0, 0);
        }
#pragma unroll
        for (int b = 0; b < NB; ++b) {
          const uint32_t w4[4] = {wv[u][b].x, wv[u][b].y, wv[u][b].z, wv[u][b].w};
          f32x4 sum[MT];
#pragma unroll
          for (int t = 0; t < MT; ++t) sum[t] = xs[t];
#pragma unroll
          for (int j = p * SPG; j < (p + 1) * SPG; ++j) {
            const bf16x8 wf = w4_values(w4[j]);
#pragma unroll
            for (int t = 0; t < MT; ++t)
              sum[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wf, as_bf16x8(xv[u][t][j]), sum[t], 0, 0, 0);
          }
          const uint2 s2 = sv[u][b][p];
          const float s4[4] = {bf2f(s2.x & 0xffff), bf2f(s2.x >> 16), bf2f(s2.y & 0xffff), bf2f(s2.y >> 16)};
#pragma unroll
          for (int t = 0; t < MT; ++t)
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[b][t][e] = fmaf(s4[e], sum[t][e], acc[b][t][e]);
        }
      }
    }
  }
  __shared__ f32x4 red[NW][NB * MT][64];
#pragma unroll
  for (int b = 0; b < NB; ++b)
#pragma unroll
    for (int t = 0; t < MT; ++t) red[wave][b * MT + t][lane] = acc[b][t];
  __syncthreads();
  for (int i = wave; i < NB * MT; i += NW) {
    f32x4 s = red[0][i][lane];
#pragma unroll
    for (int w = 1; w < NW; ++w) s += red[w][i][lane];
    w4_store(g, m0 + 16 * (i % MT) + r, (nb0 + i / MT) * 16 + 4 * q, s);
  }
}

template <int MT, int NB, int NW, int U>
hipError_t go_rows(const W4Args& g, hipStream_t s) {
  const int nbs = (g.a.N + 15) / 16;
  const dim3 grid((nbs + NB - 1) / NB, (g.a.M + 16 * MT - 1) / (16 * MT)), block(64 * NW);
  switch (g.a.group) {
    case 128: return launch((k_w4_rows<MT, NB, NW, 1, U>), grid, block, 0, s, g);
    case 64: return launch((k_w4_rows<MT, NB, NW, 2, U>), grid, block, 0, s, g);
    default: return launch((k_w4_rows<MT, NB, NW, 4, U>), grid, block, 0, s, g);
  }
}

}  // namespace

hipError_t linear_w4(const LinearW4& a, const Split& sp, hipStream_t s) {
  (void)sp;
  if (!a.x || !a.wq || !a.scales || !a.y || a.M < 1 || a.N < 1 || a.K < 32 || (a.group != 32 && a.group != 64 && a.group != 128) ||
      a.K % a.group || a.act < 0 || a.act > 2 || ((uintptr_t)a.x & 15) || (a.ldx & 7) || ((uintptr_t)a.wq & 15) ||
      ((uintptr_t)a.scales & 15) || a.ldx < a.K || a.ldy < a.N || (a.res && a.ldr < a.N))
    return hipErrorInvalidValue;
  W4Args g{};
  g.a = a;
  g.kb = (a.K + 127) / 128;
  g.groups = g.kb * (128 / a.group);
  g.vec = !((uintptr_t)a.y & (a.y_f32 ? 15 : 7)) && !(a.ldy & 3) && !((uintptr_t)a.bias & 7) && !((uintptr_t)a.res & 7) &&
          !(a.res && (a.ldr & 3));
  if (a.M <= 16) return go_rows<1, 1, 4, 4>(g, s);
  if ((a.M + 31) / 32 > 65535) return hipErrorInvalidValue;
  return go_rows<2, 1, 4, 4>(g, s);
}

}  // namespace k
}  // namespace tp
