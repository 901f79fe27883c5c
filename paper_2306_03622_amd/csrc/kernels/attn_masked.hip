// Attention with lengths, a causal order, a window and sinks (torpor_ops.h), head dim 64 or 128, on gfx950 MFMA
// (v_mfma_f32_32x32x16_bf16), one pass over the keys with a running maximum and sum per query.
//
// The query heads that share a key/value head are handled together: row rho of a sequence is head rho % G of the group at
// query rho / G (G heads per key/value head), so keys and values are read once for all of them. A workgroup
// takes 32 WR rows (WR waves of 32 side by side, each set WK waves deep over the keys) and walks tiles of 32 KPW WK
// keys through a ring of NST stages in LDS, filled by loads that go straight there (lds_load16, as in gemm_tile.hpp): rows
// as they lie in memory, their 16-byte chunks moved (k_at, v_at) so that the rows read together fall on
// different banks. One barrier per tile; keys beyond the sequence are out of the buffer's bounds and read as zeros.
//
// Scores are computed transposed, S^T = K Q^T: lane l holds row l % 32 against keys 8 (i / 4) + 4 (l / 32) + i % 4 in
// register i, so a row's maximum and sum stay in a lane and its partner l ^ 32. The output is transposed too, O^T =
// V^T P^T: the exponentials are the B operand from the very registers they are in, V^T is read with the transposing
// LDS load, and a row's rescaling is one factor per lane. For that the exponentials are rounded to bf16, as the matrix cores
// take V: a result is off by at most 2^-8 of the weights' mean of |v| for it, as much as its own rounding may add, and two
// bf16 parts of each would double V's products. The sum that divides is of the unrounded ones. The reference that exponents are taken from follows the maximum only
// when that has risen by 8 (a factor of 256, harmless in fp32 sums and in bf16, whose precision is relative).
//
// A key is seen if it lies in [lo, hi] (window and order) or in front of sk (sinks), three numbers per row. Only
// tiles that hold a key seen by some row are walked, a wave passes over those that its own rows do not see, and only those
// that they do not see whole are masked. There a score is replaced, not added to, so a hidden key may hold anything. Its value
// row, which 0 would multiply, may hold infinities or NaN: those show as NaN in the sums, and a workgroup that finds
// any such result at the end walks its keys twice more: once with what is not finite replaced by 0, and once counting,
// for each row and column, the replaced values of seen keys, which then set the output.
#include "attn_plan.hpp"
#include "gemm_tile.hpp"

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

// two bf16 with infinities and NaN as 0
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

// FAST: the hot loop. CLEAN: the same with V's infinities and NaN as zeros. COUNT: those that are seen, as sums of their kinds.
enum { FAST, CLEAN, COUNT };

template <int D, int WR, int WK, int KPW, int NST>
struct AttnTile {
  static constexpr int NW = WR * WK, KT = 32 * KPW * WK;
  static constexpr int ROW = 2 * D, CPR = ROW / 16, RPL = 1024 / ROW;          // bytes and chunks of a row, rows a load
  static constexpr int LOADS = KT / RPL / NW, LPS = 2 * LOADS;                 // of K (and of V), in all, per wave
  // what a row's 16-byte chunks are moved by: of K one chunk of 16 rows is read together, of V four chunks of 4 rows, 256 bytes
  // each time, one from each bank
  __host__ __device__ static constexpr int k_at(int row) { return D == 128 ? row % 16 : row / 2 % 8; }
  __host__ __device__ static constexpr int v_at(int row) { return D == 128 ? (row & 3) << 2 : (row & 2) << 1; }
  static constexpr int KB = KT * ROW, SBYTES = 2 * KB, DT = D / 32;
  static constexpr int REC = DT * 16 + 2;                                      // a lane's results when waves join
  static constexpr int join = (WK - 1) * WR * 64 * REC * 4, lds = NST * SBYTES > join ? NST * SBYTES : join;
  static_assert(KT % (RPL * NW) == 0 && LOADS >= 1 && KPW <= 2 && NST >= 2 && lds <= 160 * 1024, "tile shape");
};

template <int D, int WR, int WK, int KPW, int NST, int MINW>
__global__ __launch_bounds__(64 * WR * WK, MINW) void k_attention_masked(AttnArgs g) {
  typedef AttnTile<D, WR, WK, KPW, NST> T;
  constexpr int KT = T::KT, DT = T::DT;
  __shared__ __attribute__((aligned(1024))) char lds[T::lds];
  const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)lds;

  const Attention& a = g.a;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wr = wave % WR, wk = wave / WR;
  const int c = lane & 31, h = lane >> 5;
  // key/value heads first, so that workgroups handed out together read different ones and an XCD the same ones again;
  // the last rows, which see the most keys under a causal order, before the others
  int id = blockIdx.x;
  const int bh = id % (a.kv_heads * a.batch);
  id /= a.kv_heads * a.batch;
  const int z = id % g.splits, rt = g.tiles - 1 - id / g.splits;
  const int hk = bh % a.kv_heads, b = bh / a.kv_heads;

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

  // this lane's row of Q (the last one again where there is none) and what it sees; what the wave's rows see
  const bool live = row < rows;
  const int li = live ? qi : qn - 1, lh = live ? qh : hk * g.share + g.share - 1;
  const Seen me = seen_at(a, li + shift, kn);
  const int wrow = row0 + wr * 32;
  const bool idle = wrow >= rows;
  const Seen v0 = seen_at(a, wrow / g.share + shift, kn);
  const Seen v1 = seen_at(a, (min(wrow + 32, rows) - 1) / g.share + shift, kn);
  const uint16_t* qrow = a.q + (int64_t)b * a.qs[0] + (int64_t)li * a.qs[1] + (int64_t)lh * a.qs[2] + 8 * h;
  bf16x8 qf[D / 16];
#pragma unroll
  for (int i = 0; i < D / 16; ++i) qf[i] = as_bf16x8(*reinterpret_cast<const uint4*>(qrow + 16 * i));

  const uint16_t* kbase = a.k + (int64_t)b * a.ks[0] + (int64_t)hk * a.ks[2];
  const uint16_t* vbase = a.v + (int64_t)b * a.vs[0] + (int64_t)hk * a.vs[2];
  // load i of this wave: rows lrow + i RPL of a tile, at the chunk that belongs at the lane's position
  const int lrow = wave * T::LOADS * T::RPL + lane / T::CPR;
  auto issue = [&](int slot, int tile) __attribute__((always_inline)) {
    const __amdgpu_buffer_rsrc_t rk = buffer_of(kbase + (int64_t)tile * KT * a.ks[1], 0x7fffffffu);
    const __amdgpu_buffer_rsrc_t rv = buffer_of(vbase + (int64_t)tile * KT * a.vs[1], 0x7fffffffu);
    const uint32_t dst = lds0 + slot * T::SBYTES + wave * T::LOADS * 1024;
    const int left = kn - tile * KT;
#pragma unroll
    for (int i = 0; i < T::LOADS; ++i) {
      const int r = lrow + i * T::RPL;
      const uint32_t ck = (uint32_t)((lane % T::CPR) ^ T::k_at(r)) * 16, cv = (uint32_t)((lane % T::CPR) ^ T::v_at(r)) * 16;
      lds_load16<false>(rk, dst + i * 1024, r < left ? (uint32_t)r * (uint32_t)(a.ks[1] * 2) + ck : kOffNone, 0);
      lds_load16<false>(rv, dst + T::KB + i * 1024, r < left ? (uint32_t)r * (uint32_t)(a.vs[1] * 2) + cv : kOffNone, 0);
    }
  };

  f32x16 o[DT];
  float top, total;                                 // reference of the exponents (base 2), this lane's half of the sum
  const float c2 = a.scale * 1.44269504088896341f;

  // Byte addresses of this lane's fragments inside a stage, for the wave's first 32 keys: K rows, chunk 2 i + h at ka ^ 32 i; V^T
  // pieces of 4 keys x 16 columns, columns 32 t at va ^ 64 t, keys 4 h .. and 8 further.
  const uint32_t ka = (uint32_t)((wk * KPW * 32 + c) * T::ROW + ((h ^ T::k_at(c)) << 4));
  uint32_t va[2];
#pragma unroll
  for (int e = 0; e < 2; ++e) {
    const int r = wk * KPW * 32 + 8 * e + 4 * h + ((lane & 15) >> 2), ch = 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1);
    va[e] = (uint32_t)(T::KB + r * T::ROW + ((ch ^ T::v_at(r)) << 4) + (lane & 1) * 8);
  }
  // out += V^T P^T over this wave's keys of the stage at `base`
  auto values = [&](const char* base, const uint4 (&pb)[2 * KPW], f32x16 (&out)[DT]) __attribute__((always_inline)) {
#pragma unroll
    for (int u = 0; u < 2 * KPW; ++u)
#pragma unroll
      for (int t = 0; t < DT; ++t) {
        const char* p = base + 16 * u * T::ROW;
        const v4s lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) v4s*)(p + (va[0] ^ (t << 6))));
        const v4s hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) v4s*)(p + (va[1] ^ (t << 6))));
        const uint2 l2 = __builtin_bit_cast(uint2, lo), h2 = __builtin_bit_cast(uint2, hi);
        out[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(make_uint4(l2.x, l2.y, h2.x, h2.y)), as_bf16x8(pb[u]),
                                                         out[t], 0, 0, 0);
      }
  };
  // which of the 32 keys from k0 on this lane's row sees, in the order of the lane's registers: register i's key is bit
  // 8 (i / 4) + i % 4
  auto seen_bits = [&](int k0) __attribute__((always_inline)) {
    auto below = [&](int key) { return (uint32_t)((1ull << min(max(key - k0, 0), 32)) - 1); };     // keys in front of `key`
    return ((below(me.hi + 1) & ~below(me.lo)) | below(me.sk)) >> (4 * h);
  };
  auto bit_of = [](int i) { return 8 * (i >> 2) + (i & 3); };

  // scores, running maximum and sum, values of the wave's keys k0 .. of the stage at `base`
  auto attend = [&](const char* base, int k0, bool whole) __attribute__((always_inline)) {
    f32x16 sc[KPW];
#pragma unroll
    for (int u = 0; u < KPW; ++u) {
#pragma unroll
      for (int i = 0; i < D / 16; ++i)
        sc[u] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
            as_bf16x8(*reinterpret_cast<const uint4*>(base + u * 32 * T::ROW + (ka ^ (i << 5)))), qf[i],
            i == 0 ? f32x16{0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0} : sc[u], 0, 0, 0);
    }
    if (!whole) {
#pragma unroll
      for (int u = 0; u < KPW; ++u) {
        const uint32_t m = seen_bits(k0 + 32 * u);
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const uint32_t on = (uint32_t)((int32_t)(m << (31 - bit_of(i))) >> 31);        // all bits, or none
          sc[u][i] = __uint_as_float((__float_as_uint(sc[u][i]) & on) | (0xff800000u & ~on));
        }
      }
    }
    float mx = sc[0][0];
#pragma unroll
    for (int u = 0; u < KPW; ++u)
#pragma unroll
      for (int i = 0; i < 16; ++i) mx = fmaxf(mx, sc[u][i]);
    const auto half = __builtin_amdgcn_permlane32_swap(__float_as_uint(mx), __float_as_uint(mx), false, false);
    mx = fmaxf(__uint_as_float(half[0]), __uint_as_float(half[1])) * c2;                 // lanes l and l ^ 32
    if (__any(mx > top + 8.f)) {
      const float next = fmaxf(top, mx);
      const float f = next == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(top - next);
      total *= f;
#pragma unroll
      for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[d][i] *= f;
      top = next;
    }
    const float base2 = top == -INFINITY ? 0.f : top;
    uint4 pb[2 * KPW];
#pragma unroll
    for (int u = 0; u < KPW; ++u) {
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const float p = __builtin_amdgcn_exp2f(fmaf(sc[u][i], c2, -base2));
        sc[u][i] = p;
        total += p;
      }
#pragma unroll
      for (int e = 0; e < 2; ++e)
        pb[2 * u + e] = make_uint4(f2bf2(sc[u][8 * e], sc[u][8 * e + 1]), f2bf2(sc[u][8 * e + 2], sc[u][8 * e + 3]),
                                   f2bf2(sc[u][8 * e + 4], sc[u][8 * e + 5]), f2bf2(sc[u][8 * e + 6], sc[u][8 * e + 7]));
    }
    values(base, pb, o);
  };

  auto walk = [&](auto mode) __attribute__((always_inline)) {
    constexpr int MODE = decltype(mode)::value;
    top = -INFINITY;
    total = 0.f;
#pragma unroll
    for (int t = 0; t < DT; ++t)
#pragma unroll
      for (int i = 0; i < 16; ++i) o[t][i] = 0.f;
#pragma unroll
    for (int i = 0; i < NST - 1; ++i)
      if (t0 + i < t1) issue(i, w.tile(t0 + i));
    // the queries have arrived: else the compiler, which does not count the loads to LDS, waits for them (and so for the next
    // tile) in every turn of the loop
#pragma unroll
    for (int i = 0; i < D / 16; ++i) asm volatile("" : "+v"(qf[i]));
    int slot = 0;
    for (int t = t0; t < t1; ++t) {
      // tile t has landed for every wave, and the slot of tile t - 1 is free
      if (t + NST - 2 < t1) lds_wait_barrier<(NST - 2) * T::LPS>();
      else lds_wait_barrier<0>();
      if (t + NST - 1 < t1) issue(slot == 0 ? NST - 1 : slot - 1, w.tile(t + NST - 1));
      char* base = lds + slot * T::SBYTES;
      slot = slot + 1 == NST ? 0 : slot + 1;
      const int k0 = w.tile(t) * KT + wk * KPW * 32, k1 = k0 + KPW * 32;
      if constexpr (MODE != FAST) {
        for (int i = tid; i < T::KB / 16; i += 64 * T::NW) {
          uint4* p = reinterpret_cast<uint4*>(base + T::KB) + i;
          const uint4 v = *p;
          *p = MODE == CLEAN ? make_uint4(zero_odd(v.x), zero_odd(v.y), zero_odd(v.z), zero_odd(v.w))
                             : make_uint4(odd_codes(v.x), odd_codes(v.y), odd_codes(v.z), odd_codes(v.w));
        }
        __syncthreads();
      }
      if (idle || !((k0 <= v1.hi && k1 > v0.lo) || k0 < v1.sk)) continue;      // none of the wave's rows sees any
      if constexpr (MODE == COUNT) {
        f32x16 cnt[DT];
#pragma unroll
        for (int d = 0; d < DT; ++d)
#pragma unroll
          for (int i = 0; i < 16; ++i) cnt[d][i] = 0.f;
        uint4 pb[2 * KPW];
#pragma unroll
        for (int u = 0; u < 2 * KPW; ++u) {
          const uint32_t m = seen_bits(k0 + 32 * (u >> 1));
          auto one = [&](int i) __attribute__((always_inline)) { return m >> bit_of(8 * (u & 1) + i) & 1 ? 0x3f80u : 0u; };
          pb[u] = make_uint4(one(0) | one(1) << 16, one(2) | one(3) << 16, one(4) | one(5) << 16, one(6) | one(7) << 16);
        }
        values(base, pb, cnt);
#pragma unroll
        for (int d = 0; d < DT; ++d)
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const int v = (int)cnt[d][i];
            o[d][i] += ((v & 255) ? INFINITY : 0.f) - ((v >> 8 & 255) ? INFINITY : 0.f) + (v >> 16 ? NAN : 0.f);
          }
      } else {
        const bool whole = (v1.lo <= k0 && k1 - 1 <= v0.hi) || k1 <= v0.sk;
        attend(base, k0, whole);
      }
    }
    if constexpr (MODE != COUNT) total += __shfl_xor(total, 32, 64);
    if constexpr (WK > 1) {
      // the waves of one set of rows join, in wave order: counts add up, the others at a common reference
      float* area = reinterpret_cast<float*>(lds);
      __syncthreads();
      if (wk > 0) {
        float* rec = area + ((wk - 1) * WR + wr) * 64 * T::REC + lane;
        rec[0] = top;
        rec[64] = total;
#pragma unroll
        for (int d = 0; d < DT; ++d)
#pragma unroll
          for (int i = 0; i < 16; ++i) rec[(2 + d * 16 + i) * 64] = o[d][i];
      }
      __syncthreads();
      if (wk == 0) {
        float next = top;
#pragma unroll
        for (int x = 1; x < WK; ++x) next = fmaxf(next, area[((x - 1) * WR + wr) * 64 * T::REC + lane]);
        const float base2 = next == -INFINITY ? 0.f : next;
        const float f0 = MODE == COUNT ? 1.f : __builtin_amdgcn_exp2f(top - base2);
        total *= f0;
#pragma unroll
        for (int d = 0; d < DT; ++d)
#pragma unroll
          for (int i = 0; i < 16; ++i) o[d][i] *= f0;
#pragma unroll
        for (int x = 1; x < WK; ++x) {
          const float* rec = area + ((x - 1) * WR + wr) * 64 * T::REC + lane;
          const float f = MODE == COUNT ? 1.f : __builtin_amdgcn_exp2f(rec[0] - base2);
          total = fmaf(f, rec[64], total);
#pragma unroll
          for (int d = 0; d < DT; ++d)
#pragma unroll
            for (int i = 0; i < 16; ++i) o[d][i] = fmaf(f, rec[(2 + d * 16 + i) * 64], o[d][i]);
        }
        top = next;
      }
    }
    __syncthreads();
  };

  walk(std::integral_constant<int, FAST>());
  float chk = 0.f;                                  // NaN if any sum is not finite
#pragma unroll
  for (int d = 0; d < DT; ++d)
#pragma unroll
    for (int i = 0; i < 16; ++i) chk = fmaf(o[d][i], 0.f, chk);
  const bool odd = __syncthreads_or(wk == 0 && !(chk == 0.f));
  if (odd) walk(std::integral_constant<int, CLEAN>());

  // lane holds columns 32 d + 8 (i / 4) + 4 h + i % 4 of its row
  const int64_t slots = (int64_t)a.batch * a.kv_heads * all, slot = (int64_t)bh * all + row;
  float* po = g.part + (z * slots + slot) * D + 4 * h;
  if (wk == 0 && live) {
    if (g.splits > 1) {
#pragma unroll
      for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int i = 0; i < 16; i += 4)
          *reinterpret_cast<float4*>(po + 32 * d + 2 * i) = make_float4(o[d][i], o[d][i + 1], o[d][i + 2], o[d][i + 3]);
      if (h == 0)
        *reinterpret_cast<float2*>(g.part + g.splits * slots * D + (z * slots + slot) * 2) = make_float2(top, total);
    } else {
      const float inv = total == 0.f ? 0.f : 1.f / total;
#pragma unroll
      for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int i = 0; i < 16; i += 4)
          *reinterpret_cast<uint2*>(orow + 32 * d + 2 * i + 4 * h) =
              make_uint2(f2bf2(o[d][i] * inv, o[d][i + 1] * inv), f2bf2(o[d][i + 2] * inv, o[d][i + 3] * inv));
    }
  }
  if (!odd) return;
  // every seen score is -infinity: zeros, whatever the values hold (with splits the joining kernel knows)
  const bool none = g.splits == 1 && total == 0.f;
  walk(std::integral_constant<int, COUNT>());
  if (wk > 0 || !live || none) return;
#pragma unroll
  for (int d = 0; d < DT; ++d)
#pragma unroll
    for (int i = 0; i < 16; ++i)
      if (o[d][i] != 0.f) {
        const int col = 32 * d + 8 * (i >> 2) + (i & 3);
        if (g.splits > 1) po[col] += o[d][i];
        else orow[col + 4 * h] = f2bf(bf2f(orow[col + 4 * h]) + o[d][i]);
      }
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
  // lane z holds split z's maximum and sum; the values are read eight splits at a time (one split after the other,
  // 32 of them for 32 heads took 19 us)
  const float2 v = lane < g.splits ? ml[lane * slots + slot] : make_float2(-INFINITY, 0.f);
  float top = v.x;
#pragma unroll
  for (int m = 32; m > 0; m >>= 1) top = fmaxf(top, __shfl_xor(top, m, 64));
  const float f = __builtin_amdgcn_exp2f(v.x - (top == -INFINITY ? 0.f : top));
  const float total = wave_sum(f * v.y);
  float o[E] = {};
  for (int z0 = 0; z0 < g.splits; z0 += 8) {
    float p[8][E];
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
      for (int e = 0; e < E; ++e) p[i][e] = g.part[(min(z0 + i, g.splits - 1) * slots + slot) * D + lane * E + e];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float fz = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(f), min(z0 + i, 63)));
#pragma unroll
      for (int e = 0; e < E; ++e)      // an infinity (of a seen value) stays one where its split weighs next to nothing
        o[e] += z0 + i < g.splits ? (fabsf(p[i][e]) == INFINITY ? p[i][e] : fz * p[i][e]) : 0.f;
    }
  }
  const float inv = 1.f / total;
#pragma unroll
  for (int e = 0; e < E; ++e) o[e] = total == 0.f ? 0.f : o[e] * inv;          // zeros, also where an infinity was seen
  uint16_t* out = a.out + (int64_t)b * a.os[0] + (int64_t)qi * a.os[1] + (int64_t)qh * a.os[2] + lane * E;
  if constexpr (E == 2) *reinterpret_cast<uint32_t*>(out) = f2bf2(o[0], o[1]);
  else *out = f2bf(o[0]);
}

template <int D, int WR, int WK, int KPW, int NST, int MINW>
hipError_t go(AttnArgs g, hipStream_t s) {
  const int64_t rows = (int64_t)g.a.q_len * g.share;
  g.tiles = (int)((rows + 32 * WR - 1) / (32 * WR));
  const int64_t wgs = (int64_t)g.tiles * g.splits * g.a.kv_heads * g.a.batch;
  if (wgs * 64 * WR * WK >= 1ll << 32) return hipErrorInvalidValue;
  hipError_t e = launch((k_attention_masked<D, WR, WK, KPW, NST, MINW>), dim3((unsigned)wgs), dim3(64 * WR * WK), 0, s, g);
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
  // 32-bit offsets inside a tile of up to 128 keys
  if (rows * a.kv_heads * a.batch >= 1ll << 31 || a.ks[1] > 1 << 23 || a.vs[1] > 1 << 23) return hipErrorInvalidValue;
  const int64_t span = attn_span(a.q_len, a.kv_len, a.causal, a.left, a.right, a.sinks);
  const AttnPlan plan = attn_plan(a.dim, rows, (int64_t)a.kv_heads * a.batch, span, sp.partials ? sp.partial_bytes : 0);
  g.splits = plan.splits;
  g.part = sp.partials;
  switch (plan.variant) {     // dim, waves over rows and keys, 32-key blocks a wave, stages, least waves per SIMD
    case ATTN64_R32: return go<64, 1, 4, 1, 2, 2>(g, s);
    case ATTN64_R64: return go<64, 2, 2, 1, 3, 2>(g, s);
    case ATTN64_R128: return go<64, 4, 1, 1, 3, 2>(g, s);
    case ATTN64_R128_LONG: return go<64, 4, 1, 2, 2, 2>(g, s);
    case ATTN128_R32: return go<128, 1, 4, 1, 2, 1>(g, s);
    case ATTN128_R64: return go<128, 2, 2, 1, 3, 1>(g, s);
    case ATTN128_R128_DEEP: return go<128, 4, 2, 2, 2, 2>(g, s);
    case ATTN128_R128: return go<128, 4, 1, 2, 2, 2>(g, s);
    default: return go<128, 8, 1, 2, 2, 2>(g, s);
  }
}

}  // namespace k
}  // namespace tp
