// Attention with lengths, a causal order, a window and sinks (torpor_ops.h), head dim 64 or 128, on gfx950 MFMA
// (v_mfma_f32_32x32x16_bf16), one pass over the keys with a running maximum and sum per query.
//
// The query heads that share a key/value head are handled together: row rho of a sequence is head rho % G of the group at
// query rho / G (G heads per key/value head), so keys and values are read once for all of them. A workgroup
// takes 32 WR rows (WR waves of 32 side by side, each set WK waves deep over the keys) and walks tiles of 32 KPW WK
// keys, which it stages row-major in LDS; the next tile's loads are in flight meanwhile.
//
// Scores are computed transposed, S^T = K Q^T: lane l holds row l % 32 against keys 8 (i / 4) + 4 (l / 32) + i % 4 in
// register i, so a row's maximum and sum stay in a lane and its partner l ^ 32. The output is transposed too, O^T =
// V^T P^T: the exponentials, rounded to bf16 (as the matrix cores take them; the sum that divides
// them is of the unrounded ones), are the B operand from the very registers they are in, V^T is read with the transposing
// LDS load, and a row's rescaling is one factor per lane.
//
// A key is seen if it lies in [lo, hi] (window and order) or in front of sk (sinks), three numbers per row. Only
// tiles that hold a seen key are walked, and only those not seen whole by every row are masked. There a score is replaced, not
// added to, so a hidden key may hold anything; its value row, which 0 would multiply, may hold infinities or NaN: staging
// replaces those by 0 in masked tiles, and a tile that had any is followed by a second pass that counts, for each
// row and column, the replaced values of seen keys and sets the output accordingly.
#include <algorithm>

#include "common.hpp"
#include "kernels.hpp"

namespace tp {
namespace k {

struct AttnArgs {
  Attention a;
  int share;              // query heads per key/value head
  int tiles, splits;      // row tiles per (sequence, key/value head), splits over the keys
  float* part;            // splits > 1: [split][slot][dim] sums, then [split][slot][2] maximum and sum
};

template <>
struct PtrFields<AttnArgs> {
  static void add(std::vector<uint32_t>& v, uint32_t at) {
    for (size_t o : {offsetof(Attention, q), offsetof(Attention, k), offsetof(Attention, v), offsetof(Attention, out),
                     offsetof(Attention, q_lens), offsetof(Attention, kv_lens)})
      v.push_back(at + (uint32_t)(offsetof(AttnArgs, a) + o));
    v.push_back(at + (uint32_t)offsetof(AttnArgs, part));
  }
};

namespace {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef short v4s __attribute__((ext_vector_type(4)));

// the largest position a bound can reach: far beyond any length, and sums of two stay below 2^31
constexpr int kFar = 1 << 30;

// The keys that the query at position p sees: [lo, hi] and [0, sk).
struct Seen {
  int lo, hi, sk;
};
__device__ __forceinline__ Seen seen_at(const Attention& a, int p, int kn) {
  const int last = min(kn - 1, a.causal ? p : kFar);
  Seen s;
  s.lo = a.left < 0 ? 0 : max(p - a.left, 0);
  s.hi = a.right < 0 ? last : min(last, p + a.right);
  s.sk = min(a.sinks, last + 1);
  return s;
}

// A workgroup's lengths, and the key tiles of KT that its rows [row0, row1) see: sink tiles [0, ns), then [w0, w1).
struct Walk {
  int qn, kn, ns, w0, w1;
  __device__ __forceinline__ int count() const { return ns + max(0, w1 - w0); }
  __device__ __forceinline__ int tile(int t) const { return t < ns ? t : w0 + t - ns; }
};

// bit pattern of a bf16 infinity or NaN in the low or high half
__device__ __forceinline__ bool odd_half(uint32_t w) {
  return (w & 0x7f80u) == 0x7f80u || (w & 0x7f800000u) == 0x7f800000u;
}
__device__ __forceinline__ uint32_t zero_odd(uint32_t w) {
  if ((w & 0x7f80u) == 0x7f80u) w &= 0xffff0000u;
  if ((w & 0x7f800000u) == 0x7f800000u) w &= 0xffffu;
  return w;
}
// the code of a bf16 in the counting pass: +infinity 1, -infinity 256, NaN 65536, anything else 0
__device__ __forceinline__ uint32_t odd_code(uint32_t h) {
  if ((h & 0x7f80u) != 0x7f80u) return 0;
  return (h & 0x7fu) ? 0x4780u : (h & 0x8000u) ? 0x4380u : 0x3f80u;
}
__device__ __forceinline__ uint32_t odd_codes(uint32_t w) { return odd_code(w & 0xffff) | odd_code(w >> 16) << 16; }

template <int D, int WR, int WK, int KPW>
__global__ __launch_bounds__(64 * WR * WK) void k_attention_masked(AttnArgs g) {
  constexpr int NT = 64 * WR * WK, KT = 32 * KPW * WK;
  constexpr int LDK = D + 8, LDV = D + 16;          // row strides in LDS: reads of 16 rows fall on different banks
  constexpr int CH = D / 8, NL = KT * CH / NT;      // 16-byte pieces of a key, loads per thread and tile
  constexpr int DT = D / 32;
  static_assert(KT * CH % NT == 0, "whole loads");
  constexpr int KV = (LDK + LDV) * KT * 2, MERGE = WK > 1 ? (WK - 1) * WR * 64 * (DT * 16 + 2) * 4 : 0;
  __shared__ __attribute__((aligned(16))) char lds[KV > MERGE ? KV : MERGE];
  __shared__ int odd[2];                            // of the tiles by turns, see the loop
  uint16_t* Ks = reinterpret_cast<uint16_t*>(lds);
  uint16_t* Vs = Ks + LDK * KT;

  const Attention& a = g.a;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int wr = wave % WR, wk = wave / WR;
  const int c = lane & 31, h = lane >> 5;
  int id = blockIdx.x;
  const int z = id % g.splits;
  id /= g.splits;
  const int rt = id % g.tiles;
  id /= g.tiles;
  const int hk = id % a.kv_heads, b = id / a.kv_heads;

  int qn = a.q_lens ? a.q_lens[b] : a.q_len, kn = a.kv_lens ? a.kv_lens[b] : a.kv_len;
  qn = min(max(qn, 0), a.q_len);
  kn = min(max(kn, 0), a.kv_len);
  const int rows = qn * g.share, row0 = rt * 32 * WR, all = a.q_len * g.share;
  const int row = row0 + wr * 32 + c;               // this lane's row
  const int qi = row / g.share, qh = hk * g.share + row - qi * g.share;
  uint16_t* orow = a.out + (int64_t)b * a.os[0] + (int64_t)qi * a.os[1] + (int64_t)qh * a.os[2];
  if (a.zero_tail && z == 0 && wk == 0 && row >= rows && row < all) {
    for (int i = 0; i < D / 16; ++i) *reinterpret_cast<uint4*>(orow + h * (D / 2) + 8 * i) = make_uint4(0, 0, 0, 0);
  }
  if (row0 >= rows) return;

  const int shift = kn - qn;                        // query i stands at i + shift
  const Seen s0 = seen_at(a, row0 / g.share + shift, kn);
  const Seen s1 = seen_at(a, (min(row0 + 32 * WR, rows) - 1) / g.share + shift, kn);
  Walk w;
  w.ns = s1.sk > 0 ? (s1.sk + KT - 1) / KT : 0;
  w.w0 = max(s0.lo / KT, w.ns);
  w.w1 = s1.hi >= s0.lo ? s1.hi / KT + 1 : 0;
  const int n = w.count();
  const int t0 = (int)((int64_t)n * z / g.splits), t1 = (int)((int64_t)n * (z + 1) / g.splits);

  // this lane's row of Q (the last one again where there is none) and what it sees
  const bool live = row < rows;
  const int li = live ? qi : qn - 1, lh = live ? qh : hk * g.share + g.share - 1;
  const Seen me = seen_at(a, li + shift, kn);
  const uint16_t* qrow = a.q + (int64_t)b * a.qs[0] + (int64_t)li * a.qs[1] + (int64_t)lh * a.qs[2] + 8 * h;
  uint4 qf[D / 16];
#pragma unroll
  for (int i = 0; i < D / 16; ++i) qf[i] = *reinterpret_cast<const uint4*>(qrow + 16 * i);

  const uint16_t* kbase = a.k + (int64_t)b * a.ks[0] + (int64_t)hk * a.ks[2];
  const uint16_t* vbase = a.v + (int64_t)b * a.vs[0] + (int64_t)hk * a.vs[2];
  uint4 kr[NL], vr[NL];
  // keys beyond the sequence are not read and count as zero
  auto load = [&](int tile) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < NL; ++i) {
      const int at = i * NT + tid, key = tile * KT + at / CH, d = (at % CH) * 8;
      kr[i] = vr[i] = make_uint4(0, 0, 0, 0);
      if (key < kn) {
        kr[i] = *reinterpret_cast<const uint4*>(kbase + (int64_t)key * a.ks[1] + d);
        vr[i] = *reinterpret_cast<const uint4*>(vbase + (int64_t)key * a.vs[1] + d);
      }
    }
  };

  f32x16 o[DT];
#pragma unroll
  for (int t = 0; t < DT; ++t)
#pragma unroll
    for (int i = 0; i < 16; ++i) o[t][i] = 0.f;
  float top = -INFINITY, total = 0.f;               // maximum (in base-2 exponents), this lane's half of the sum
  const float c2 = a.scale * 1.44269504088896341f;

  // V^T P^T for this wave's keys of the tile in LDS
  const uint16_t* vread = Vs + (wk * KPW * 32 + 4 * h + ((lane & 15) >> 2)) * LDV + 16 * ((lane >> 4) & 1) + 4 * (lane & 3);
  auto values = [&](const uint4 (&pb)[2 * KPW], f32x16 (&out)[DT]) __attribute__((always_inline)) {
#pragma unroll
    for (int u = 0; u < 2 * KPW; ++u)
#pragma unroll
      for (int t = 0; t < DT; ++t) {
        const uint16_t* p = vread + 16 * u * LDV + 32 * t;
        const v4s lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) v4s*)p);
        const v4s hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) v4s*)(p + 8 * LDV));
        const uint2 l2 = __builtin_bit_cast(uint2, lo), h2 = __builtin_bit_cast(uint2, hi);
        out[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(make_uint4(l2.x, l2.y, h2.x, h2.y)), as_bf16x8(pb[u]),
                                                         out[t], 0, 0, 0);
      }
  };

  if (tid < 2) odd[tid] = 0;
  if (t0 < t1) load(w.tile(t0));
  for (int t = t0; t < t1; ++t) {
    const int tile = w.tile(t), k0 = tile * KT;
    // seen whole by every row: inside the window of the first and the last, or among the sinks
    const bool whole = (s1.lo <= k0 && k0 + KT - 1 <= s0.hi) || k0 + KT <= s0.sk;
    bool mine = false;
#pragma unroll
    for (int i = 0; i < NL; ++i) {
      const int at = i * NT + tid, key = at / CH, d = (at % CH) * 8;
      uint4 v = vr[i];
      if (!whole) {
        const bool any = odd_half(v.x) || odd_half(v.y) || odd_half(v.z) || odd_half(v.w);
        if (any) v = make_uint4(zero_odd(v.x), zero_odd(v.y), zero_odd(v.z), zero_odd(v.w));
        mine = mine || any;
      }
      *reinterpret_cast<uint4*>(Ks + key * LDK + d) = kr[i];
      *reinterpret_cast<uint4*>(Vs + key * LDV + d) = v;
    }
    __syncthreads();
    // set between a tile's two barriers and read behind the second; the next tile's flag, last read before the
    // first, is cleared in the same place
    if (mine) odd[t & 1] = 1;
    if (tid == 0) odd[(t + 1) & 1] = 0;
    if (t + 1 < t1) load(w.tile(t + 1));

    f32x16 sc[KPW];
#pragma unroll
    for (int u = 0; u < KPW; ++u) {
#pragma unroll
      for (int i = 0; i < 16; ++i) sc[u][i] = 0.f;
      const uint16_t* kread = Ks + ((wk * KPW + u) * 32 + c) * LDK + 8 * h;
#pragma unroll
      for (int i = 0; i < D / 16; ++i)
        sc[u] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(*reinterpret_cast<const uint4*>(kread + 16 * i)),
                                                        as_bf16x8(qf[i]), sc[u], 0, 0, 0);
    }
    uint32_t sees = 0xffffffffu;                    // bit 16 u + i: register i of block u is a seen key
    static_assert(KPW <= 2, "one bit per score");
    if (!whole) {
      sees = 0;
#pragma unroll
      for (int u = 0; u < KPW; ++u)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const int key = k0 + (wk * KPW + u) * 32 + 8 * (i >> 2) + 4 * h + (i & 3);
          const bool yes = (key >= me.lo && key <= me.hi) || key < me.sk;
          sc[u][i] = yes ? sc[u][i] : -INFINITY;
          sees |= yes ? 1u << (16 * u + i) : 0u;
        }
    }
    float mx = sc[0][0];
#pragma unroll
    for (int u = 0; u < KPW; ++u)
#pragma unroll
      for (int i = 0; i < 16; ++i) mx = fmaxf(mx, sc[u][i]);
    mx = fmaxf(mx, __shfl_xor(mx, 32, 64)) * c2;
    if (__any(mx > top)) {
      const float next = fmaxf(top, mx);
      const float f = next == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(top - next);
      total *= f;
#pragma unroll
      for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[d][i] *= f;
      top = next;
    }
    const float base = top == -INFINITY ? 0.f : top;
    uint4 pb[2 * KPW];
#pragma unroll
    for (int u = 0; u < KPW; ++u) {
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const float p = __builtin_amdgcn_exp2f(fmaf(sc[u][i], c2, -base));
        sc[u][i] = p;
        total += p;
      }
#pragma unroll
      for (int e = 0; e < 2; ++e)
        pb[2 * u + e] = make_uint4(f2bf2(sc[u][8 * e], sc[u][8 * e + 1]), f2bf2(sc[u][8 * e + 2], sc[u][8 * e + 3]),
                                   f2bf2(sc[u][8 * e + 4], sc[u][8 * e + 5]), f2bf2(sc[u][8 * e + 6], sc[u][8 * e + 7]));
    }
    values(pb, o);
    __syncthreads();
    if (!whole && odd[t & 1]) {
      // the tile's value rows held infinities or NaN: their codes take the place of V, the seen keys' ones that of P
#pragma unroll 1
      for (int i = 0; i < NL; ++i) {
        const int at = i * NT + tid, key = tile * KT + at / CH, d = (at % CH) * 8;
        uint4 v = make_uint4(0, 0, 0, 0);
        if (key < kn) v = *reinterpret_cast<const uint4*>(vbase + (int64_t)key * a.vs[1] + d);
        *reinterpret_cast<uint4*>(Vs + (at / CH) * LDV + d) =
            make_uint4(odd_codes(v.x), odd_codes(v.y), odd_codes(v.z), odd_codes(v.w));
      }
      __syncthreads();
      f32x16 cnt[DT];
#pragma unroll
      for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) cnt[d][i] = 0.f;
#pragma unroll
      for (int u = 0; u < 2 * KPW; ++u) {
        const uint32_t m = sees >> (8 * u);
        auto pair = [&](int i) { return ((m >> i) & 1 ? 0x3f80u : 0u) | ((m >> (i + 1)) & 1 ? 0x3f800000u : 0u); };
        pb[u] = make_uint4(pair(0), pair(2), pair(4), pair(6));
      }
      values(pb, cnt);
#pragma unroll
      for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const int v = (int)cnt[d][i];
          const bool plus = v & 255, minus = (v >> 8) & 255;
          if (v >= 65536 || (plus && minus)) o[d][i] = NAN;
          else if (plus) o[d][i] += INFINITY;
          else if (minus) o[d][i] -= INFINITY;
        }
      __syncthreads();
    }
  }

  total += __shfl_xor(total, 32, 64);
  if constexpr (WK > 1) {
    // the waves of one set of rows join: maxima and sums first, then the outputs, in wave order
    float* area = reinterpret_cast<float*>(lds);
    constexpr int REC = DT * 16 + 2;
    __syncthreads();
    if (wk > 0) {
      float* rec = area + ((wk - 1) * WR + wr) * 64 * REC + lane;
      rec[0] = top;
      rec[64] = total;
#pragma unroll
      for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) rec[(2 + d * 16 + i) * 64] = o[d][i];
    }
    __syncthreads();
    if (wk > 0) return;
    float next = top;
#pragma unroll
    for (int x = 1; x < WK; ++x) next = fmaxf(next, area[((x - 1) * WR + wr) * 64 * REC + lane]);
    const float base = next == -INFINITY ? 0.f : next;
    const float f0 = __builtin_amdgcn_exp2f(top - base);
    total *= f0;
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
      for (int i = 0; i < 16; ++i) o[d][i] *= f0;
#pragma unroll
    for (int x = 1; x < WK; ++x) {
      const float* rec = area + ((x - 1) * WR + wr) * 64 * REC + lane;
      const float f = __builtin_amdgcn_exp2f(rec[0] - base);
      total = fmaf(f, rec[64], total);
#pragma unroll
      for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[d][i] = fmaf(f, rec[(2 + d * 16 + i) * 64], o[d][i]);
    }
    top = next;
  }
  if (!live) return;
  // lane holds columns 32 d + 8 (i / 4) + 4 h + i % 4 of its row
  if (g.splits > 1) {
    const int64_t slots = (int64_t)a.batch * a.kv_heads * all, slot = ((int64_t)b * a.kv_heads + hk) * all + row;
    float* po = g.part + (z * slots + slot) * D + 4 * h;
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
      for (int i = 0; i < 16; i += 4)
        *reinterpret_cast<float4*>(po + 32 * d + 2 * i) = make_float4(o[d][i], o[d][i + 1], o[d][i + 2], o[d][i + 3]);
    if (h == 0)
      *reinterpret_cast<float2*>(g.part + g.splits * slots * D + (z * slots + slot) * 2) = make_float2(top, total);
    return;
  }
  const float inv = total == 0.f ? 0.f : 1.f / total;
#pragma unroll
  for (int d = 0; d < DT; ++d)
#pragma unroll
    for (int i = 0; i < 16; i += 4)
      *reinterpret_cast<uint2*>(orow + 32 * d + 2 * i + 4 * h) =
          make_uint2(f2bf2(o[d][i] * inv, o[d][i + 1] * inv), f2bf2(o[d][i + 2] * inv, o[d][i + 3] * inv));
}

// Joins the splits of a row in split order: a wave per row.
template <int D>
__global__ __launch_bounds__(256) void k_attention_join(AttnArgs g) {
  constexpr int E = D / 64;
  const Attention& a = g.a;
  const int lane = threadIdx.x & 63;
  const int64_t slot = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  const int all = a.q_len * g.share;
  const int64_t slots = (int64_t)a.batch * a.kv_heads * all;
  if (slot >= slots) return;
  const int row = (int)(slot % all);
  const int64_t bh = slot / all;
  const int hk = (int)(bh % a.kv_heads), b = (int)(bh / a.kv_heads);
  const int qn = a.q_lens ? min(max(a.q_lens[b], 0), a.q_len) : a.q_len;
  const int qi = row / g.share, qh = hk * g.share + row - qi * g.share;
  if (qi >= qn) return;
  const float2* ml = reinterpret_cast<const float2*>(g.part + g.splits * slots * D);
  float top = -INFINITY;
  for (int z = 0; z < g.splits; ++z) top = fmaxf(top, ml[z * slots + slot].x);
  const float base = top == -INFINITY ? 0.f : top;
  float total = 0.f, o[E] = {};
  for (int z = 0; z < g.splits; ++z) {
    const float2 v = ml[z * slots + slot];
    const float f = __builtin_amdgcn_exp2f(v.x - base);
    total = fmaf(f, v.y, total);
    const float* p = g.part + (z * slots + slot) * D + lane * E;
#pragma unroll
    for (int e = 0; e < E; ++e) o[e] = fmaf(f, p[e], o[e]);
  }
  const float inv = total == 0.f ? 0.f : 1.f / total;
  uint16_t* out = a.out + (int64_t)b * a.os[0] + (int64_t)qi * a.os[1] + (int64_t)qh * a.os[2] + lane * E;
  if constexpr (E == 2) *reinterpret_cast<uint32_t*>(out) = f2bf2(o[0] * inv, o[1] * inv);
  else *out = f2bf(o[0] * inv);
}

template <int D, int WR, int WK, int KPW>
hipError_t go(AttnArgs g, hipStream_t s) {
  const int64_t rows = (int64_t)g.a.q_len * g.share;
  g.tiles = (int)((rows + 32 * WR - 1) / (32 * WR));
  const int64_t wgs = (int64_t)g.tiles * g.splits * g.a.kv_heads * g.a.batch;
  if (wgs * 64 * WR * WK >= 1ll << 32) return hipErrorInvalidValue;
  hipError_t e = launch((k_attention_masked<D, WR, WK, KPW>), dim3((unsigned)wgs), dim3(64 * WR * WK), 0, s, g);
  if (e != hipSuccess || g.splits == 1) return e;
  const int64_t slots = rows * g.a.kv_heads * g.a.batch;
  return launch((k_attention_join<D>), dim3((unsigned)((slots + 3) / 4)), dim3(256), 0, s, g);
}

// A wave per sequence, four ids a lane and step.
__global__ __launch_bounds__(256) void k_seq_lengths(const int32_t* __restrict__ ids, int B, int S, int32_t* __restrict__ lens) {
  const int lane = threadIdx.x & 63, b = blockIdx.x * 4 + (threadIdx.x >> 6);
  if (b >= B) return;
  const int32_t* row = ids + (int64_t)b * S;
  int first = S;
  for (int s0 = 0; s0 < S && first == S; s0 += 256) {
    int at = S;
#pragma unroll
    for (int i = 3; i >= 0; --i) {
      const int s = s0 + 64 * i + lane;
      const unsigned long long neg = __ballot(s < S && row[min(s, S - 1)] < 0);
      if (neg) at = s0 + 64 * i + __builtin_ctzll(neg);
    }
    first = at;
  }
  if (lane == 0) lens[b] = first;
}

}  // namespace

hipError_t seq_lengths(const int32_t* ids, int B, int S, int32_t* lens, hipStream_t s) {
  if (!ids || !lens || B < 1 || S < 1) return hipErrorInvalidValue;
  return launch(k_seq_lengths, dim3((B + 3) / 4), dim3(256), 0, s, ids, B, S, lens);
}

hipError_t attention_masked(const Attention& a, const Split& sp, hipStream_t s) {
  if (!a.q || !a.out || (a.kv_len > 0 && (!a.k || !a.v)) || a.batch < 1 || a.q_len < 1 || a.kv_len < 0 || a.kv_heads < 1 || a.heads < 1 ||
      a.heads % a.kv_heads || (a.dim != 64 && a.dim != 128) || !(a.scale > 0.f))
    return hipErrorInvalidValue;
  AttnArgs g{};
  g.a = a;
  g.share = a.heads / a.kv_heads;
  const int64_t rows = (int64_t)a.q_len * g.share;
  if (rows * a.kv_heads * a.batch >= 1ll << 31) return hipErrorInvalidValue;
  // few rows: the keys are split over workgroups too
  const int wr = rows > 32 ? 4 : 1, kt = wr == 4 ? 64 : 128;
  const int64_t base = (rows + 32 * wr - 1) / (32 * wr) * a.kv_heads * a.batch;
  int64_t span = a.kv_len;
  if (a.left >= 0 && (a.causal || a.right >= 0))
    span = std::min<int64_t>(span, (int64_t)a.left + (a.causal ? 0 : a.right) + std::min<int64_t>(a.q_len, 32 * wr) + a.sinks);
  const int64_t tiles = (span + kt - 1) / kt;
  const int64_t slots = rows * a.kv_heads * a.batch, fits = (int64_t)(sp.partials ? sp.partial_bytes / 4 : 0) / (slots * (a.dim + 2));
  int64_t z = std::min<int64_t>({512 / base, tiles / 2, fits, 128});
  g.splits = (int)std::max<int64_t>(z, 1);
  g.part = sp.partials;
  if (a.dim == 64) return wr == 4 ? go<64, 4, 1, 2>(g, s) : go<64, 1, 4, 1>(g, s);
  return wr == 4 ? go<128, 4, 1, 2>(g, s) : go<128, 1, 4, 1>(g, s);
}

}  // namespace k
}  // namespace tp
