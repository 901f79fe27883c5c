// Attention of a few new tokens over a paged cache (torpor_serve.h), head dim 64 or 128, values bf16 or e4m3, on gfx950
// MFMA (v_mfma_f32_16x16x32_bf16), one pass over the keys with a running maximum and sum per query.
//
// The query heads that share a key/value head are handled together: row rho of a sequence is head rho % G of the group at
// query rho / G, so keys and values are read once for all of them. A workgroup takes 16 RB rows and a stretch of tiles of 32 keys; its
// waves take the tiles in turns and do not wait for each other: each has a ring of NST tiles in LDS of its own, filled by
// loads that go straight there, and waits for its own loads alone. At the end the waves join through LDS, and
// workgroups that split a sequence's keys through `work` in a second launch.
//
// A page holds at least 16 tokens, so each half of a tile lies in one page: its number comes by a scalar load, and the
// half's place goes into a buffer resource that ends behind the sequence's last key (and is empty for an entry that is no
// page), so that what lies behind reads as zeros and no lane checks anything. Rows in LDS lie as in memory, their
// 16-byte chunks moved (k_at, v_at) so that the rows read together fall on different banks.
//
// Scores are computed transposed, S^T = K Q^T: lane l holds row l % 16 against keys 4 (l / 16) + i of each half. The
// exponentials, in bf16 as the matrix cores take V, are then the next product's operand where they are, if its
// 32 keys are taken in that order: O^T = V^T P^T, with V^T read by the transposing LDS loads in the same order of keys. They go in as two
// bf16 parts (rest_of), so that 2^-15 of each is lost: with one, the error against 64 bits was 0.0021 to 0.0023 (norm over norm), where the
// result's rounding alone gives 0.0017; the second takes 1 to 4% of a call (24 tokens over up to 4096 66.1 -> 66.8 us, 64 over up to 500 22.8 -> 23.4, 8 new tokens of two sequences over up to 20,000 in
// 8 bits 27.8 -> 29.9). 8-bit keys
// become bf16 exactly, times their scale, as they are read (v_cvt_scalef32_pk_bf16_fp8); 8-bit values become bf16
// without it, and their scale multiplies the exponential before that is taken apart (scale byte 255, NaN to the conversion, is an infinite
// factor there, whose rest is NaN). The sum that divides is of the exponentials as they are.
// The reference that exponents are taken from follows the maximum only when that has risen by 8 (a factor of 256, harmless in
// fp32 sums and in bf16, whose precision is relative).
//
// A hidden key's score is replaced, not added to, and its exponential is 0; its value row, which the matrix cores would
// multiply by that, may hold anything. Where a tile holds hidden keys and a value that is not finite, its values are added one by one,
// those of seen keys only. So whatever lies behind a window's edge or a drafted token's stays out.
#include "gemm_tile.hpp"
#include "serve_args.hpp"
#include "cache_plan.hpp"

namespace tp {
namespace k {

struct CacheAttnArgs {
  CacheAttention a;
  int share;              // query heads per key/value head
  int tiles, splits;      // row tiles per (sequence, key/value head), splits over the keys
  float* part;            // splits > 1: [split][slot][dim] sums, then [split][slot][2] maximum and sum
};

namespace {

typedef short v4s __attribute__((ext_vector_type(4)));
typedef int v2i __attribute__((ext_vector_type(2)));
#define LDS_PTR(T, p) ((__attribute__((address_space(3))) T*)(p))

// Loads straight into LDS, as lds_load16 (gemm_tile.hpp): lane l's 16 or 4 bytes land at `dst` + their size times l. The
// buffer's description may come from a vector instruction (v_readfirstlane, or v_readlane where the compiler keeps scalars in
// a vector register), and a load needs five wait states behind one that writes the scalars it reads; the compiler does
// not see the load, so the block holds them (without: keys of the wrong half, in a kernel that had three in between).
__device__ __forceinline__ void to_lds16(__amdgpu_buffer_rsrc_t r, uint32_t dst, uint32_t voff) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(dst), "v"(voff), "s"(r) : "m0");
}
__device__ __forceinline__ void to_lds4(__amdgpu_buffer_rsrc_t r, uint32_t dst, uint32_t voff) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tbuffer_load_dword %1, %2, 0 offen lds" ::"s"(dst), "v"(voff), "s"(r) : "m0");
}
// This wave's LDS reads so far have returned: what they read may be written over.
__device__ __forceinline__ void reads_done() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }
// At most N of this wave's loads are in flight.
template <int N>
__device__ __forceinline__ void loads_left() { asm volatile("s_waitcnt vmcnt(%0)" ::"i"(N) : "memory"); }

// A buffer whose place and size are the same for the wave but were computed in vector registers.
__device__ __forceinline__ __amdgpu_buffer_rsrc_t buffer_at(const char* p, int bytes) {
  const uint64_t at = (uint64_t)(uintptr_t)p;
  const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)at), hi = __builtin_amdgcn_readfirstlane((uint32_t)(at >> 32));
  return buffer_of(reinterpret_cast<const void*>((uintptr_t)((uint64_t)hi << 32 | lo)), (uint32_t)__builtin_amdgcn_readfirstlane(bytes));
}

// An exponential's first bf16 part is its leading bits, the second what is left, rounded. 2^-23 of the exponential is added to that, in
// the same operation: so the rest of a positive one is positive too, and an infinite value times both parts is that infinity.
__device__ __forceinline__ uint32_t first_parts(float lo, float hi) { return __builtin_amdgcn_perm(__float_as_uint(hi), __float_as_uint(lo), 0x07060302u); }
__device__ __forceinline__ float rest_of(float p) { return fmaf(p, 0x1.000002p0f, -__uint_as_float(__float_as_uint(p) & 0xffff0000u)); }

// The keys that the query at position p sees: [lo, hi] and [0, sk).
struct Seen {
  int lo, hi, sk;
};
__device__ __forceinline__ Seen seen_at(const CacheAttention& a, int p, int kn) {
  Seen s;
  s.hi = min(kn - 1, p);
  s.lo = a.window < 0 ? 0 : max(p - a.window, 0);
  s.sk = min(a.sinks, s.hi + 1);
  return s;
}

template <int D, bool E4M3, int NST>
struct Ring {
  static constexpr int ROW = E4M3 ? D : 2 * D, CPR = ROW / 16, RPL = 1024 / ROW;   // bytes and chunks of a row, rows a load
  static constexpr int HL = 16 / RPL;                                            // loads of half a tile's keys
  static constexpr int KB = 32 * ROW, SBYTES = 2 * KB + (E4M3 ? 256 : 0);        // a tile's keys, a stage
  static constexpr int LPS = 4 * HL + (E4M3 ? 1 : 0);                            // loads a stage
  // What a row's chunks are moved by. K: one chunk of 16 rows is read together (half a chunk at a time for e4m3, both
  // halves in turn); V: bf16 two chunks of 8 rows, e4m3 one chunk of rows r .. r + 7 and 16 + r ...
  __device__ static constexpr int k_at(int r) { return ROW == 256 ? r % 16 : ROW == 128 ? r / 2 % 8 : r / 4 % 4; }
  __device__ static constexpr int v_at(int r) {
    return E4M3 ? (ROW == 128 ? (r / 2 % 4) | (r / 16 % 2) << 2 : (r / 4 % 2) | (r / 16 % 2) << 1) : ROW == 256 ? r % 8 << 1 : r / 2 % 4 << 1;
  }
  static_assert(16 % RPL == 0 && (NST - 1) * LPS < 64, "ring shape");
};

template <int D, bool E4M3, int RB, int W, int NST>
__global__ __launch_bounds__(64 * W) void k_cache_attention(CacheAttnArgs g) {
  typedef Ring<D, E4M3, NST> T;
  constexpr int DT = D / 16, DC = D / 32;           // column tiles of the output, products a score takes
  constexpr int REC = RB * (DT * 4 + 2);            // a lane's results when waves join
  constexpr int RING = NST * T::SBYTES, JOIN = (W - 1) * 64 * REC * 4, LDS = W * RING > JOIN ? W * RING : JOIN;
  static_assert(LDS <= 160 * 1024, "LDS");
  __shared__ __attribute__((aligned(1024))) char lds[LDS];

  const CacheAttention& a = g.a;
  const Cache& c = a.c;
  const int tid = threadIdx.x, lane = tid & 63, r16 = lane & 15, q4 = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  int id = blockIdx.x;
  const int bh = id % (c.heads * a.p.batch);
  id /= c.heads * a.p.batch;
  const int z = id % g.splits, rt = id / g.splits;
  const int hk = bh % c.heads, b = bh / c.heads;

  // What does not wait for the lengths is asked for beside them: Q's rows (the last one again where there is none; a row that has
  // no query is computed and not stored) and, for keys from the first on, the pages of this wave's first tiles.
  const int row0 = rt * 16 * RB, all = a.p.q_len * g.share;
  bf16x8 qf[RB][DC];
#pragma unroll
  for (int rb = 0; rb < RB; ++rb) {
    const int row = min(row0 + rb * 16 + r16, all - 1), qi = row / g.share, qh = hk * g.share + row - qi * g.share;
    const uint16_t* p = a.q + b * a.qs[0] + qi * a.qs[1] + qh * a.qs[2];
#pragma unroll
    for (int i = 0; i < DC; ++i)      // e4m3 keys come 16 columns a lane, for two products
      qf[rb][i] = as_bf16x8(*reinterpret_cast<const uint4*>(p + (E4M3 ? 64 * (i / 2) + 16 * q4 + 8 * (i % 2) : 32 * i + 8 * q4)));
  }
  const auto* table = (const __attribute__((address_space(4))) int32_t*)(uintptr_t)(a.p.table + b * a.p.table_stride);
  auto page_at = [&](int t, int hb) __attribute__((always_inline)) { return table[min((t * 32 + hb * 16) >> c.lg, a.p.max_pages - 1)]; };
  const bool from0 = a.window < 0 && g.splits == 1;
  int early[NST - 1][2];
#pragma unroll
  for (int i = 0; i < NST - 1; ++i)
#pragma unroll
    for (int hb = 0; hb < 2; ++hb) early[i][hb] = page_at(wave + i * W, hb);
  const Lens len = lens_of(a.p, b);
  const int qn = len.qn, kn = min(len.kn, a.kv_len), rows = qn * g.share;
  if (row0 >= rows) return;
  const int shift = kn - qn;                        // query i stands at i + shift
  const int row1 = min(row0 + 16 * RB, rows) - 1;
  const Seen first = seen_at(a, row0 / g.share + shift, kn), last = seen_at(a, row1 / g.share + shift, kn);
  // tiles that hold a key seen by some row: sinks [0, ns), then [w0, w1)
  const int ns = last.sk > 0 ? (last.sk + 31) / 32 : 0, w0 = max(first.lo / 32, ns), w1 = last.hi >= first.lo ? last.hi / 32 + 1 : 0;
  const int n = ns + max(0, w1 - w0);
  const int t0 = (int)((int64_t)n * z / g.splits), t1 = (int)((int64_t)n * (z + 1) / g.splits);
  auto tile = [&](int t) __attribute__((always_inline)) { return t < ns ? t : w0 + t - ns; };

  Seen me[RB];                                      // what this lane's rows see
#pragma unroll
  for (int rb = 0; rb < RB; ++rb) me[rb] = seen_at(a, min(row0 + rb * 16 + r16, rows - 1) / g.share + shift, kn);

  char* ring = lds + wave * RING;
  const uint32_t ring0 = (uint32_t)(uintptr_t)LDS_PTR(char, lds) + wave * RING;
  const char *kp = static_cast<const char*>(c.k) + hk * c.ks[2], *vp = static_cast<const char*>(c.v) + hk * c.vs[2];
  const int mask = (1 << c.lg) - 1;
  uint32_t gone = 0;                                // two bits a stage under way, the youngest lowest: halves in no page
  const int lr = lane / T::CPR, lc = lane % T::CPR;
  // Loads tile `t`, in these pages, into a slot: K's halves, V's halves, exponents.
  auto issue = [&](int slot, int t, int page0, int page1) __attribute__((always_inline)) {
    const uint32_t dst = ring0 + slot * T::SBYTES;
    uint32_t xoff[2];
    gone <<= 2;
#pragma unroll
    for (int hb = 0; hb < 2; ++hb) {
      const int key = __builtin_amdgcn_readfirstlane(t * 32 + hb * 16), at = key & mask;
      int page = hb ? page1 : page0;
      const bool ok = (unsigned)page < (unsigned)c.pages && key >> c.lg < a.p.max_pages;
      const int rows = ok ? min(max(kn - key, 0), 16) : 0;
      page = ok ? page : 0;
      gone |= (ok ? 0u : 1u) << hb;
      const uint32_t krow = (uint32_t)c.ks[1], vrow = (uint32_t)c.vs[1];
      const __amdgpu_buffer_rsrc_t rk = buffer_at(kp + page * c.ks[0] + at * c.ks[1], rows ? (rows - 1) * krow + T::ROW : 0);
      const __amdgpu_buffer_rsrc_t rv = buffer_at(vp + page * c.vs[0] + at * c.vs[1], rows ? (rows - 1) * vrow + T::ROW : 0);
#pragma unroll
      for (int i = 0; i < T::HL; ++i) {
        const int r = i * T::RPL + lr;
        const uint32_t to = dst + (hb * T::HL + i) * 1024;
        to_lds16(rk, to, r * krow + (uint32_t)(lc ^ T::k_at(hb * 16 + r)) * 16);
        to_lds16(rv, to + T::KB, r * vrow + (uint32_t)(lc ^ T::v_at(hb * 16 + r)) * 16);
      }
      xoff[hb] = rows ? (uint32_t)((page * 2 * c.heads + hk) << c.lg) + at : kOffNone;
    }
    if constexpr (E4M3) {
      // lanes 0..7: K's exponents of keys 4 l .., lanes 8..15: V's (bytes 0..31 and 32..63 of the stage's last 256)
      const uint32_t half = lane & 4 ? xoff[1] : xoff[0];
      const uint32_t off = half + 4 * (lane & 3) + (lane & 8 ? (uint32_t)(c.heads << c.lg) : 0u);
      to_lds4(buffer_of(c.exps, (uint32_t)(c.pages * 2 * c.heads) << c.lg), dst + 2 * T::KB, lane < 16 && half != kOffNone ? off : kOffNone);
    }
  };

  f32x4 o[RB][DT];
  float top[RB], total[RB];                         // reference of the exponents (base 2), this lane's quarter of the sum
  const float c2 = a.scale * 1.44269504088896341f;
#pragma unroll
  for (int rb = 0; rb < RB; ++rb) {
    top[rb] = -INFINITY;
    total[rb] = 0.f;
#pragma unroll
    for (int t = 0; t < DT; ++t) o[rb][t] = f32x4{0, 0, 0, 0};
  }

  // Scores, running maximum and sum, values of the tile at `base`, whose keys start at k0; lost: halves in no page.
  auto attend = [&](const char* base, int k0, uint32_t lost) __attribute__((always_inline)) {
    f32x4 s[RB][2];
#pragma unroll
    for (int hb = 0; hb < 2; ++hb) {
      const int r = hb * 16 + r16;
      const char* row = base + r * T::ROW;
      bf16x8 kf[DC];
      if constexpr (E4M3) {
        const float f = __uint_as_float((uint32_t)(uint8_t)base[2 * T::KB + r] << 23);
#pragma unroll
        for (int i = 0; i < DC; i += 2) {
          const uint4 w = *reinterpret_cast<const uint4*>(row + (((2 * i + q4) ^ T::k_at(r)) << 4));
          auto eight = [&](uint32_t x, uint32_t y) {
            uint4 e;
            e.x = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x, f, false));
            e.y = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x, f, true));
            e.z = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(y, f, false));
            e.w = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(y, f, true));
            return as_bf16x8(e);
          };
          kf[i] = eight(w.x, w.y);
          kf[i + 1] = eight(w.z, w.w);
        }
      } else {
#pragma unroll
        for (int i = 0; i < DC; ++i)
          kf[i] = as_bf16x8(*reinterpret_cast<const uint4*>(row + (((4 * i + q4) ^ T::k_at(r)) << 4)));
      }
#pragma unroll
      for (int rb = 0; rb < RB; ++rb)
#pragma unroll
        for (int i = 0; i < DC; ++i)
          s[rb][hb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[i], qf[rb][i], i ? s[rb][hb] : f32x4{0, 0, 0, 0}, 0, 0, 0);
    }
    const bool whole = !lost && ((last.lo <= k0 && k0 + 31 <= first.hi) || k0 + 31 < first.sk);
    uint32_t on[RB];                                // bit 4 hb + i: this lane's key 16 hb + 4 q4 + i is seen
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) on[rb] = 0xffu;
    if (!whole) {
      const uint32_t held = (lost & 1 ? 0u : 0x0fu) | (lost & 2 ? 0u : 0xf0u);
      auto below = [&](int key) {                   // this lane's keys in front of `key`
        const uint32_t m = (uint32_t)((1ull << min(max(key - k0 - 4 * q4, 0), 32)) - 1);
        return (m & 0xfu) | (m >> 12 & 0xf0u);
      };
#pragma unroll
      for (int rb = 0; rb < RB; ++rb) {
        on[rb] = ((below(me[rb].hi + 1) & ~below(me[rb].lo)) | below(me[rb].sk)) & held;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const uint32_t keep = (uint32_t)((int32_t)(on[rb] << (31 - i)) >> 31);         // all bits, or none
          s[rb][i / 4][i % 4] = __uint_as_float((__float_as_uint(s[rb][i / 4][i % 4]) & keep) | (0xff800000u & ~keep));
        }
      }
    }
    float vs[2][4];
    if constexpr (E4M3) {
#pragma unroll
      for (int hb = 0; hb < 2; ++hb) {
        const uint32_t x = *reinterpret_cast<const uint32_t*>(base + 2 * T::KB + 32 + 16 * hb + 4 * q4);
#pragma unroll
        for (int i = 0; i < 4; ++i) vs[hb][i] = __uint_as_float(max((x >> (8 * i) & 255u) << 23, 0x400000u));         // byte 0: 2^-127
      }
    }
    uint4 pb[RB], pr[RB];                           // first parts, rests
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
      float mx = s[rb][0][0];
#pragma unroll
      for (int i = 1; i < 8; ++i) mx = fmaxf(mx, s[rb][i / 4][i % 4]);
      const auto h16 = __builtin_amdgcn_permlane16_swap(__float_as_uint(mx), __float_as_uint(mx), false, false);
      mx = fmaxf(__uint_as_float(h16[0]), __uint_as_float(h16[1]));
      const auto h32 = __builtin_amdgcn_permlane32_swap(__float_as_uint(mx), __float_as_uint(mx), false, false);
      mx = fmaxf(__uint_as_float(h32[0]), __uint_as_float(h32[1])) * c2;               // lanes of the same row
      if (__any(mx > top[rb] + 8.f)) {
        const float next = fmaxf(top[rb], mx);
        const float f = next == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(top[rb] - next);
        total[rb] *= f;
#pragma unroll
        for (int t = 0; t < DT; ++t) o[rb][t] *= f;
        top[rb] = next;
      }
      const float ref = top[rb] == -INFINITY ? 0.f : top[rb];
      float p[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        p[i] = __builtin_amdgcn_exp2f(fmaf(s[rb][i / 4][i % 4], c2, -ref));
        total[rb] += p[i];
        if constexpr (E4M3) p[i] = on[rb] >> i & 1 ? p[i] * vs[i / 4][i % 4] : 0.f;    // (a hidden key's scale may be infinite)
      }
      pb[rb] = make_uint4(first_parts(p[0], p[1]), first_parts(p[2], p[3]), first_parts(p[4], p[5]), first_parts(p[6], p[7]));
      pr[rb] = make_uint4(f2bf2(rest_of(p[0]), rest_of(p[1])), f2bf2(rest_of(p[2]), rest_of(p[3])), f2bf2(rest_of(p[4]), rest_of(p[5])),
                          f2bf2(rest_of(p[6]), rest_of(p[7])));
    }
    if (!whole) {
      bool odd = false;                             // a value that is not finite
#pragma unroll
      for (int i = 0; i < T::KB / 1024; ++i) {
        const uint4 w = *reinterpret_cast<const uint4*>(base + T::KB + i * 1024 + lane * 16);
        for (uint32_t x : {w.x, w.y, w.z, w.w}) {
          if constexpr (E4M3) {
#pragma unroll
            for (int e = 0; e < 32; e += 8) odd |= (x >> e & 0x7fu) == 0x7fu;
          } else {
            odd |= (x & 0x7f80u) == 0x7f80u || (x & 0x7f800000u) == 0x7f800000u;
          }
        }
      }
      if (__any(odd)) {
#pragma unroll
        for (int rb = 0; rb < RB; ++rb)
          for (int key = 0; key < 32; ++key) {
            const int i = 4 * (key >> 4) + (key & 3), from = 16 * (key >> 2 & 3) + r16;
            // (by value: a choice among places in memory would put the parts into LDS, in every tile)
            auto part = [&](uint32_t x, uint32_t y, uint32_t z, uint32_t w) {
              const uint32_t lo = i < 2 ? x : y, hi = i < 6 ? z : w, two = (uint32_t)__shfl((int)(i < 4 ? lo : hi), from, 64);
              return __uint_as_float(i & 1 ? two & 0xffff0000u : two << 16);
            };
            const float p = part(pb[rb].x, pb[rb].y, pb[rb].z, pb[rb].w) + part(pr[rb].x, pr[rb].y, pr[rb].z, pr[rb].w);
            const bool see = (uint32_t)__shfl((int)on[rb], from, 64) >> i & 1;
            const char* row = base + T::KB + key * T::ROW;
#pragma unroll
            for (int t = 0; t < DT; ++t) {
              float v[4];
              if constexpr (E4M3) {
                const uint32_t x = *reinterpret_cast<const uint32_t*>(row + ((t ^ T::v_at(key)) << 4) + 4 * q4);
                const uint32_t lo = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x, 1.f, false));
                const uint32_t hi = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x, 1.f, true));
                v[0] = __uint_as_float(lo << 16), v[1] = __uint_as_float(lo & 0xffff0000u);
                v[2] = __uint_as_float(hi << 16), v[3] = __uint_as_float(hi & 0xffff0000u);
              } else {
                const uint2 x = *reinterpret_cast<const uint2*>(row + (((2 * t + (q4 >> 1)) ^ T::v_at(key)) << 4) + 8 * (q4 & 1));
                v[0] = __uint_as_float(x.x << 16), v[1] = __uint_as_float(x.x & 0xffff0000u);
                v[2] = __uint_as_float(x.y << 16), v[3] = __uint_as_float(x.y & 0xffff0000u);
              }
#pragma unroll
              for (int e = 0; e < 4; ++e) o[rb][t][e] += see ? p * v[e] : 0.f;
            }
          }
        return;
      }
    }
    // O^T += V^T P^T: columns 16 t + r16, keys 4 q4 .. and 16 + 4 q4 ..
#pragma unroll
    for (int t = 0; t < DT; ++t) {
      bf16x8 vf;
      if constexpr (E4M3) {
        const int j = r16 >> 1, key = j < 4 ? 4 * q4 + j : 12 + 4 * q4 + j;
        const v2i w = __builtin_amdgcn_ds_read_tr8_b64_v2i32(LDS_PTR(v2i, base + T::KB + key * T::ROW + ((t ^ T::v_at(key)) << 4) + 8 * (r16 & 1)));
        vf = as_bf16x8(make_uint4(__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w.x, 1.f, false)),
                                  __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w.x, 1.f, true)),
                                  __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w.y, 1.f, false)),
                                  __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w.y, 1.f, true))));
      } else {
        const int key = 4 * q4 + (r16 >> 2), ch = 2 * t + (r16 >> 1 & 1);
        const char* p = base + T::KB + key * T::ROW + 8 * (r16 & 1);
        const v4s lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16(LDS_PTR(v4s, p + ((ch ^ T::v_at(key)) << 4)));
        const v4s hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16(LDS_PTR(v4s, p + 16 * T::ROW + ((ch ^ T::v_at(key + 16)) << 4)));
        const uint2 l2 = __builtin_bit_cast(uint2, lo), h2 = __builtin_bit_cast(uint2, hi);
        vf = as_bf16x8(make_uint4(l2.x, l2.y, h2.x, h2.y));
      }
#pragma unroll
      for (int rb = 0; rb < RB; ++rb) {
        o[rb][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, as_bf16x8(pb[rb]), o[rb][t], 0, 0, 0);
        o[rb][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, as_bf16x8(pr[rb]), o[rb][t], 0, 0, 0);
      }
    }
  };

  // this wave's tiles: t0 + wave, every W-th
  const int mine = t1 - t0 > wave ? (t1 - t0 - wave + W - 1) / W : 0;
  auto mine_at = [&](int i) __attribute__((always_inline)) { return tile(t0 + wave + i * W); };
#pragma unroll
  for (int i = 0; i < NST - 1; ++i)
    if (i < mine) issue(i, mine_at(i), from0 ? early[i][0] : page_at(mine_at(i), 0), from0 ? early[i][1] : page_at(mine_at(i), 1));
  // the queries have arrived: else the compiler, which does not count the loads to LDS, waits for them in the loop
#pragma unroll
  for (int rb = 0; rb < RB; ++rb)
#pragma unroll
    for (int i = 0; i < DC; ++i) asm volatile("" : "+v"(qf[rb][i]));
  int slot = 0;
  for (int i = 0; i < mine; ++i) {
    reads_done();
    uint32_t lost;
    if (i + NST - 1 < mine) {
      const int t = mine_at(i + NST - 1);
      issue(slot == 0 ? NST - 1 : slot - 1, t, page_at(t, 0), page_at(t, 1));
      loads_left<(NST - 1) * T::LPS>();
      lost = gone >> (2 * (NST - 1)) & 3;
    } else {
      loads_left<0>();
      lost = gone >> (2 * (mine - 1 - i)) & 3;
    }
    attend(ring + slot * T::SBYTES, mine_at(i) * 32, lost);
    slot = slot + 1 == NST ? 0 : slot + 1;
  }
#pragma unroll
  for (int rb = 0; rb < RB; ++rb) {
    total[rb] += __shfl_xor(total[rb], 16, 64);
    total[rb] += __shfl_xor(total[rb], 32, 64);
  }

  if constexpr (W > 1) {
    // the waves join in their order, at a common reference
    float* area = reinterpret_cast<float*>(lds);
    __syncthreads();
    if (wave > 0) {
      float* rec = area + (wave - 1) * 64 * REC + lane;
#pragma unroll
      for (int rb = 0; rb < RB; ++rb) {
        *rec = top[rb], rec[64] = total[rb];
        rec += 128;
#pragma unroll
        for (int t = 0; t < DT; ++t)
#pragma unroll
          for (int e = 0; e < 4; ++e) *rec = o[rb][t][e], rec += 64;
      }
    }
    __syncthreads();
    if (wave > 0) return;
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
      const float* rec = area + rb * 64 * (DT * 4 + 2) + lane;
      float next = top[rb];
#pragma unroll
      for (int x = 0; x < W - 1; ++x) next = fmaxf(next, rec[x * 64 * REC]);
      const float ref = next == -INFINITY ? 0.f : next;
      const float f0 = __builtin_amdgcn_exp2f(top[rb] - ref);
      total[rb] *= f0;
#pragma unroll
      for (int t = 0; t < DT; ++t) o[rb][t] *= f0;
#pragma unroll
      for (int x = 0; x < W - 1; ++x) {
        const float f = __builtin_amdgcn_exp2f(rec[x * 64 * REC] - ref);
        total[rb] = fmaf(f, rec[x * 64 * REC + 64], total[rb]);
#pragma unroll
        for (int t = 0; t < DT; ++t)
#pragma unroll
          for (int e = 0; e < 4; ++e) o[rb][t][e] = fmaf(f, rec[x * 64 * REC + (2 + t * 4 + e) * 64], o[rb][t][e]);
      }
      top[rb] = next;
    }
  }

  // lane holds columns 16 t + 4 q4 + e of its rows
#pragma unroll
  for (int rb = 0; rb < RB; ++rb) {
    const int row = row0 + rb * 16 + r16;
    if (row >= rows) continue;
    if (g.splits > 1) {
      const int64_t slots = (int64_t)a.p.batch * c.heads * all, slot_at = z * slots + (int64_t)bh * all + row;
#pragma unroll
      for (int t = 0; t < DT; ++t)
        *reinterpret_cast<float4*>(g.part + slot_at * D + 16 * t + 4 * q4) = make_float4(o[rb][t][0], o[rb][t][1], o[rb][t][2], o[rb][t][3]);
      if (q4 == 0) *reinterpret_cast<float2*>(g.part + g.splits * slots * D + slot_at * 2) = make_float2(top[rb], total[rb]);
    } else {
      const int qi = row / g.share, qh = hk * g.share + row - qi * g.share;
      uint16_t* orow = a.out + b * a.os[0] + qi * a.os[1] + qh * a.os[2];
      const bool none = total[rb] == 0.f;           // zeros, whatever the values hold
      const float inv = 1.f / total[rb];
#pragma unroll
      for (int t = 0; t < DT; ++t)
        *reinterpret_cast<uint2*>(orow + 16 * t + 4 * q4) =
            none ? make_uint2(0, 0) : make_uint2(f2bf2(o[rb][t][0] * inv, o[rb][t][1] * inv), f2bf2(o[rb][t][2] * inv, o[rb][t][3] * inv));
    }
  }
}

// Joins the splits of a row in split order: a wave per row, or WIDE a workgroup, whose waves take 16 splits each. All that it reads, the
// first 16 splits' sums among it, is asked for at once; what belongs to a row that has no query is read and dropped (one read behind
// the other took 4.7 us for two splits).
template <int D, bool WIDE>
__global__ __launch_bounds__(256) void k_cache_join(CacheAttnArgs g) {
  constexpr int E = D / 64, Z = 16;
  __shared__ float sums[WIDE ? 3 : 1][E][64];
  const CacheAttention& a = g.a;
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), first = WIDE ? wave * Z : 0;
  const int64_t slot = WIDE ? (int64_t)blockIdx.x : (int64_t)blockIdx.x * 4 + wave;
  const int all = a.p.q_len * g.share;
  const int64_t slots = (int64_t)a.p.batch * a.c.heads * all;
  if (slot >= slots) return;
  const int row = (int)(slot % all);
  const int64_t bh = slot / all;
  const int hk = (int)(bh % a.c.heads), b = (int)(bh / a.c.heads);
  const int qi = row / g.share, qh = hk * g.share + row - qi * g.share;
  const float2* ml = reinterpret_cast<const float2*>(g.part + g.splits * slots * D);
  const int live = a.p.q_lens ? a.p.q_lens[b] : a.p.q_len;
  // lane z holds split z's maximum and sum
  const float2 v = lane < g.splits ? ml[lane * slots + slot] : make_float2(-INFINITY, 0.f);
  float p[Z][E];
  auto load = [&](int z0) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < Z; ++i)
#pragma unroll
      for (int e = 0; e < E; ++e) p[i][e] = z0 + i < g.splits ? g.part[((z0 + i) * slots + slot) * D + lane * E + e] : 0.f;
  };
  load(first);
  if (qi >= live) return;                           // (WIDE: the whole workgroup)
  float top = v.x;
#pragma unroll
  for (int m = 32; m > 0; m >>= 1) top = fmaxf(top, __shfl_xor(top, m, 64));
  const float f = __builtin_amdgcn_exp2f(v.x - (top == -INFINITY ? 0.f : top));
  const float total = wave_sum(f * v.y);
  float o[E] = {};
  for (int z0 = first; z0 < (WIDE ? first + 1 : g.splits); z0 += Z) {
    if (!WIDE && z0) load(z0);
#pragma unroll
    for (int i = 0; i < Z; ++i) {
      const float fz = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(f), min(z0 + i, 63)));
#pragma unroll
      for (int e = 0; e < E; ++e) o[e] += z0 + i < g.splits ? fz * p[i][e] : 0.f;
    }
  }
  if constexpr (WIDE) {
    if (wave > 0)
#pragma unroll
      for (int e = 0; e < E; ++e) sums[wave - 1][e][lane] = o[e];
    __syncthreads();
    if (wave > 0) return;
#pragma unroll
    for (int w = 0; w < 3; ++w)
#pragma unroll
      for (int e = 0; e < E; ++e) o[e] += sums[w][e][lane];
  }
  const float inv = 1.f / total;
#pragma unroll
  for (int e = 0; e < E; ++e) o[e] = total == 0.f ? 0.f : o[e] * inv;
  uint16_t* out = a.out + b * a.os[0] + qi * a.os[1] + qh * a.os[2] + lane * E;
  if constexpr (E == 2) *reinterpret_cast<uint32_t*>(out) = f2bf2(o[0], o[1]);
  else *out = f2bf(o[0]);
}

template <int D, bool E4M3, int RB, int W, int NST>
hipError_t go(CacheAttnArgs g, hipStream_t s) {
  const int64_t rows = (int64_t)g.a.p.q_len * g.share, heads = (int64_t)g.a.c.heads * g.a.p.batch;
  g.tiles = (int)((rows + 16 * RB - 1) / (16 * RB));
  const int64_t wgs = heads * g.tiles * g.splits;
  if (wgs * 64 * W >= 1ll << 32) return hipErrorInvalidValue;
  hipError_t e = launch((k_cache_attention<D, E4M3, RB, W, NST>), dim3((unsigned)wgs), dim3(64 * W), 0, s, g);
  if (e != hipSuccess || g.splits == 1) return e;
  // A workgroup per row where its splits are more than a wave asks for at once, and rows few (us, a wave / a workgroup, with exponentials in
  // one part: one token of 8 heads on one, 64 values, over 60,000 21.6 / 15.5, with two 15.9; two of 4096 11.0 / 9.4; one of 32 heads over 100,001 in 8 bits 49.7 / 48.7).
  if (g.splits > 16 && rows * heads <= 4096) return launch((k_cache_join<D, true>), dim3((unsigned)(rows * heads)), dim3(256), 0, s, g);
  return launch((k_cache_join<D, false>), dim3((unsigned)((rows * heads + 3) / 4)), dim3(256), 0, s, g);
}

template <int D, bool E4M3>
hipError_t by_rows(const CacheAttnArgs& g, const CachePlan& plan, hipStream_t s) {
  const int rb = plan.rb;
  constexpr int NST = D == 64 ? 3 : 2;
  if (rb == 1 && plan.waves == 1) return go<D, E4M3, 1, 1, 2>(g, s);
  if (rb == 1 && plan.waves == 2) return go<D, E4M3, 1, 2, NST>(g, s);
  return rb == 1 ? go<D, E4M3, 1, 4, NST>(g, s) : rb == 2 ? go<D, E4M3, 2, 4, NST>(g, s) : go<D, E4M3, 4, 4, NST>(g, s);
}

}  // namespace

hipError_t cache_attention(const CacheAttention& a, const Split& sp, hipStream_t s) {
  const Cache& c = a.c;
  if (!c.k || !c.v || (c.e4m3 && !c.exps) || !a.p.table || !a.p.kv_lens || !a.q || !a.out || (c.dim != 64 && c.dim != 128) || a.p.batch < 1 ||
      a.p.q_len < 1 || c.heads < 1 || a.heads < 1 || a.heads % c.heads || c.pages < 1 || a.p.max_pages < 1 || c.lg < 4 || c.lg > 12 ||
      a.kv_len < 0 || !(a.scale > 0.f))
    return hipErrorInvalidValue;
  CacheAttnArgs g{};
  g.a = a;
  g.share = a.heads / c.heads;
  const int64_t rows = (int64_t)a.p.q_len * g.share, heads = (int64_t)c.heads * a.p.batch;
  if (rows * heads >= 1 << 27) return hipErrorInvalidValue;
  const int64_t span = cache_span(a.p.q_len, a.kv_len, a.window, a.sinks);
  const CachePlan plan = cache_plan(c.dim, c.e4m3, rows, heads, span, a.p.batch == 1 || span <= a.kv_len / 2, sp.partials ? sp.partial_bytes : 0);
  g.splits = plan.splits;
  g.part = sp.partials;
  if (c.dim == 64) return c.e4m3 ? by_rows<64, true>(g, plan, s) : by_rows<64, false>(g, plan, s);
  return c.e4m3 ? by_rows<128, true>(g, plan, s) : by_rows<128, false>(g, plan, s);
}

}  // namespace k
}  // namespace tp
