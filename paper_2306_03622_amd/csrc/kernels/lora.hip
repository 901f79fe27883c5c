// Low-rank adapters of many requests beside a shared projection (torpor_serve.h): y[m] = act(base[m] + s_a B_a (A_a x[m])),
// a = adapter[m], on gfx950 MFMA (v_mfma_f32_16x16x32_bf16).
//
// Two launches: k_lora_down computes t = s A x (fp32, in `work`), k_lora_up adds B t to the base. In both a workgroup (or wave) takes a tile of
// rows, finds the adapters that they name (the rows' numbers lie one in a lane; a ballot gives an adapter's rows), and takes
// the rows of one adapter together, in blocks of 16, wherever in the tile they stand: rows of many requests in any order need no
// sorting, and no row meets another's adapter. Where there are few tiles, the adapters of a tile go to several workgroups.
// Where many tiles could hold many adapters each, k_lora_order first writes down the rows adapter by adapter, and tiles are of that order;
// where a tile holds few, one more workgroup of k_lora_down does so for k_lora_up.
// Without scratch k_lora does both in one launch and computes t anew for every 256 outputs; where scratch holds t of a part of the rows, they are
// taken part by part (lora_rows).
//
// t is taken as bf16 parts (two, three for fp32 results: 2^-16 and 2^-24 of t), all multiplied by B, whose values are bf16 as they are.
// Operands: A's rows r against x's rows m (t^T), then t's rows m against B's rows n, those of four blocks interleaved so
// that a lane ends with four consecutive outputs of a row. What lies behind a rank is not used, whatever it holds.
#include "lora_plan.hpp"
#include "serve_args.hpp"

namespace tp {
namespace k {

struct LoraArgs {
  Lora a;
  float* t;               // [splits][M][R]
  int2* order;            // [M] rows and their adapters (-1: none), adapter by adapter; NULL: as they stand
  int2* order_out;        // what one more workgroup of the first product writes for the second, or NULL
  int splits;             // over K
  int slots;              // workgroups (or waves) that share a tile's adapters
  int tiles_n;            // blocks of outputs
  int run, xcds;          // second product: blocks of 64 outputs a workgroup, XCDs that tiles are handed to
};

namespace {

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

__device__ __forceinline__ uint4 zeros() { return make_uint4(0, 0, 0, 0); }
__device__ __forceinline__ uint4 load16(const void* p) { return *reinterpret_cast<const uint4*>(p); }

// bf16 pairs of a chunk of eight values, those from `n` on as zeros
__device__ __forceinline__ uint4 first_of(uint4 v, int n) {
  uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int j = 0; j < 4; ++j) w[j] &= n >= 2 * j + 2 ? 0xffffffffu : n == 2 * j + 1 ? 0xffffu : 0u;
  return make_uint4(w[0], w[1], w[2], w[3]);
}

__device__ __forceinline__ int rank_of(const Lora& a, int ad) { return a.ranks ? min(max(a.ranks[ad], 0), a.R) : a.R; }

// The rest of t behind its bf16 part (none behind an infinity or NaN).
__device__ __forceinline__ float rest_of(float t, uint16_t part) { return fabsf(t) < INFINITY ? t - bf2f(part) : 0.f; }

// A lane's four consecutive outputs of a row as one vector, at any multiple of their element (one access on this hardware; as
// single elements 3444 rows of 3592 x 5702, rank 128, took 119 us, so 87).
typedef u32x2 u32x2_at2 __attribute__((aligned(2)));
typedef u32x4 u32x4_at4 __attribute__((aligned(4)));

// The base's values there, loaded ahead (m: a row that is there; outputs behind N are not used).
template <bool F32, bool STREAM>
struct Base {
  uint4 w;                // fp32, or bf16 pairs in x and y
  __device__ __forceinline__ void load(const Lora& a, int64_t m, int n) {
    w = zeros();
    if (!a.base || n >= a.N) return;
    const int64_t at = m * a.ldbase + n;
    const int last = a.N - 1 - n;                   // the last one again behind N
    if constexpr (F32) {
      const uint32_t* p = static_cast<const uint32_t*>(a.base) + at;
      if (last >= 3) {
        const u32x4_at4* q = reinterpret_cast<const u32x4_at4*>(p);
        u32x4 u;
        if constexpr (STREAM) u = __builtin_nontemporal_load(q);
        else u = *q;
        w = make_uint4(u.x, u.y, u.z, u.w);
      } else {
        w = make_uint4(p[0], p[min(1, last)], p[min(2, last)], 0);
      }
    } else {
      const uint16_t* p = static_cast<const uint16_t*>(a.base) + at;
      if (last >= 3) {
        const u32x2_at2* q = reinterpret_cast<const u32x2_at2*>(p);
        u32x2 u;
        if constexpr (STREAM) u = __builtin_nontemporal_load(q);
        else u = *q;
        w.x = u.x, w.y = u.y;
      } else {
        w.x = p[0] | (uint32_t)p[min(1, last)] << 16, w.y = p[min(2, last)];
      }
    }
  }
  __device__ __forceinline__ f32x4 values() const {
    if constexpr (F32) return __builtin_bit_cast(f32x4, w);
    return f32x4{__uint_as_float(w.x << 16), __uint_as_float(w.x & 0xffff0000u), __uint_as_float(w.y << 16), __uint_as_float(w.y & 0xffff0000u)};
  }
};

// The activation of all of a lane's results: one choice for them, so that their chains of operations overlap.
template <int R>
__device__ __forceinline__ void activate(f32x4 (&v)[R], int act) {
  if (act == ACT_RELU) {
#pragma unroll
    for (int i = 0; i < 4 * R; ++i) v[i / 4][i % 4] = v[i / 4][i % 4] < 0.f ? 0.f : v[i / 4][i % 4];           // keeps NaN
  } else if (act == ACT_GELU) {
#pragma unroll
    for (int i = 0; i < 4 * R; ++i) v[i / 4][i % 4] = act_apply(v[i / 4][i % 4], ACT_GELU);
  }
}

// Row m's four outputs.
template <bool F32, bool STREAM>
__device__ __forceinline__ void store(const Lora& a, int64_t m, int n, f32x4 v) {
  const int64_t at = m * a.ldy + n;
  if (n <= a.N - 4) {
    if constexpr (F32) {
      u32x4_at4* p = reinterpret_cast<u32x4_at4*>(static_cast<float*>(a.y) + at);
      if constexpr (STREAM) __builtin_nontemporal_store(__builtin_bit_cast(u32x4_at4, v), p);
      else *p = __builtin_bit_cast(u32x4_at4, v);
    } else {
      const u32x2_at2 w = {f2bf2(v[0], v[1]), f2bf2(v[2], v[3])};
      u32x2_at2* p = reinterpret_cast<u32x2_at2*>(static_cast<uint16_t*>(a.y) + at);
      if constexpr (STREAM) __builtin_nontemporal_store(w, p);
      else *p = w;
    }
    return;
  }
#pragma unroll
  for (int j = 0; j < 3; ++j) {
    if (n + j >= a.N) continue;
    if constexpr (F32) static_cast<float*>(a.y)[at + j] = v[j];
    else static_cast<uint16_t*>(a.y)[at + j] = f2bf(v[j]);
  }
}

__device__ __forceinline__ int adapter_of(const Lora& a, int row) {
  const int id = a.adapter[row];
  return (unsigned)id < (unsigned)a.adapters ? id : -1;
}

// The row at place m0 + lane of a tile of ROWS (lanes behind it, and places behind the last: row m0) and its adapter (-1: none).
template <int ROWS>
__device__ __forceinline__ int2 place_of(const LoraArgs& g, int m0, int lane) {
  const bool real = lane < ROWS && m0 + lane < g.a.M;
  if (g.order) {
    const int2 p = g.order[real ? m0 + lane : m0];
    return make_int2(p.x, real ? p.y : -1);
  }
  return make_int2(real ? m0 + lane : m0, real ? adapter_of(g.a, m0 + lane) : -1);
}

// Lane j holds the number of the j-th set bit of `mask` (behind the last: 0).
__device__ __forceinline__ int nth_of(unsigned long long mask, int lane) {
  const int before = (int)__builtin_amdgcn_mbcnt_hi((uint32_t)(mask >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)mask, 0));
  // lanes without a bit send to lane 63, where the last bit's lane sends too if all 64 are set: then no lane is without
  return __builtin_amdgcn_ds_permute((mask >> lane & 1 ? before : 63) * 4, mask >> lane & 1 ? lane : 0);
}

// The rows adapter by adapter, those without one last: counted, summed up, and put in their places. Where 64 rows side by side
// have the same one they go by one addition and keep their order; else an adapter's rows are in no fixed order, since a row's result does not
// depend on its place. One workgroup: 8192 rows take 8 us.
constexpr int kMostBins = 4096;

__global__ __launch_bounds__(1024) void k_lora_order(LoraArgs g) {
  __shared__ int bins[kMostBins], sums[16];
  const Lora& a = g.a;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, n = a.adapters + 1;
  for (int i = tid; i < n; i += 1024) bins[i] = 0;
  __syncthreads();
  // adds one to each row's bin, a wave's rows together where they have the same one, and gives what was there before
  auto take = [&](int bin, bool real) __attribute__((always_inline)) {
    const unsigned long long mask = __ballot(real);
    if (!mask) return 0;
    const int lead = (int)__builtin_ctzll(mask), b = __builtin_amdgcn_readlane(bin, lead);
    if (__ballot(real && bin == b) != mask) return real ? atomicAdd(&bins[bin], 1) : 0;
    int first = 0;
    if (lane == lead) first = atomicAdd(&bins[b], __builtin_popcountll(mask));
    return __builtin_amdgcn_readlane(first, lead) + (int)__builtin_amdgcn_mbcnt_hi((uint32_t)(mask >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)mask, 0));
  };
  // goes through the rows, eight of a thread's asked for at once
  constexpr int AHEAD = 8;
  auto each_row = [&](auto use) __attribute__((always_inline)) {
    for (int m0 = tid; m0 - tid < a.M; m0 += 1024 * AHEAD) {
      int id[AHEAD];
#pragma unroll
      for (int i = 0; i < AHEAD; ++i) id[i] = m0 + 1024 * i < a.M ? a.adapter[m0 + 1024 * i] : -1;
#pragma unroll
      for (int i = 0; i < AHEAD; ++i) {
        if ((unsigned)id[i] >= (unsigned)a.adapters) id[i] = -1;
        const int m = m0 + 1024 * i;
        if (m - tid < a.M) use(m, id[i], take(id[i] < 0 ? n - 1 : id[i], m < a.M));
      }
    }
  };
  each_row([](int, int, int) {});
  __syncthreads();
  // each thread's four bins, then the lanes of a wave, then the waves
  constexpr int EACH = kMostBins / 1024;
  int mine[EACH], sum = 0;
#pragma unroll
  for (int i = 0; i < EACH; ++i) {
    const int at = tid * EACH + i;
    mine[i] = sum;
    sum += at < n ? bins[at] : 0;
  }
  int upto = sum;
#pragma unroll
  for (int step = 1; step < 64; step *= 2) {
    const int before = __shfl_up(upto, step, 64);
    if (lane >= step) upto += before;
  }
  if (lane == 63) sums[wave] = upto;
  __syncthreads();
  int base = upto - sum;
  for (int w = 0; w < wave; ++w) base += sums[w];
#pragma unroll
  for (int i = 0; i < EACH; ++i)
    if (tid * EACH + i < n) bins[tid * EACH + i] = base + mine[i];
  __syncthreads();
  each_row([&](int m, int id, int at) {
    if (m < a.M) g.order[at] = make_int2(m, id);
  });
}

// Workgroups are handed out to the eight XCDs in turn: tiles side by side, whose rows often have the same adapter, for one XCD.
__device__ __forceinline__ int tile_of(int id, int tiles) {
  const int each = tiles >> 3, more = tiles & 7, x = id & 7;
  return x * each + min(x, more) + (id >> 3);
}

// The same order for up to seven adapters and kLoraFewRows rows, by one workgroup of W waves: every lane has a run of rows, whose
// bins (the adapter, or none) lie in LDS a byte each; it counts them in eight packed counters, the counts are summed up over the lanes
// before, and it puts its rows in their places. Every adapter's rows keep their order.
template <int W>
__device__ __forceinline__ void order_few(const Lora& a, int2* order, char* lds, int wave, int lane) {
  constexpr int T = 64 * W, AHEAD = 8, kSums = 20 * 1024;
  static_assert(kLoraFew < 8 && kLoraFewRows + 4 * 2 * T <= kSums && kLoraFewRows < 1 << 15, "packed counters");
  const int tid = wave * 64 + lane, none = a.adapters, words = ((a.M + 4 * T - 1) / (4 * T)) | 1;      // of a lane; odd: no bank conflicts
  for (int m0 = tid; m0 - tid < words * 4 * T; m0 += T * AHEAD) {
    int id[AHEAD];
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) id[i] = a.adapter[min(m0 + i * T, a.M - 1)];
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) {
      const int m = m0 + i * T;
      if (m < words * 4 * T) lds[m] = m >= a.M ? 8 : (unsigned)id[i] < (unsigned)none ? (char)id[i] : (char)none;
    }
  }
  __syncthreads();
  const uint32_t* mine = reinterpret_cast<const uint32_t*>(lds) + tid * words;
  // 16 bits a bin, four to a word
  uint64_t lo = 0, hi = 0;
  for (int i = 0; i < words; ++i)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const uint32_t bin = mine[i] >> (8 * e) & 255u;
      const uint64_t one = 1ull << (16 * (bin & 3));
      lo += bin < 4 ? one : 0;
      hi += bin >= 4 && bin < 8 ? one : 0;
    }
  uint64_t lo_to = lo, hi_to = hi;                  // of the lanes up to this one
#pragma unroll
  for (int step = 1; step < 64; step *= 2) {
    const uint64_t l = __shfl_up(lo_to, step, 64), h = __shfl_up(hi_to, step, 64);
    if (lane >= step) lo_to += l, hi_to += h;
  }
  uint64_t* sums = reinterpret_cast<uint64_t*>(lds + kSums);
  if (lane == 63) sums[2 * wave] = lo_to, sums[2 * wave + 1] = hi_to;
  __syncthreads();
  uint64_t lo_all = 0, hi_all = 0;
  lo_to -= lo, hi_to -= hi;
#pragma unroll
  for (int w = 0; w < W; ++w) {
    lo_all += sums[2 * w], hi_all += sums[2 * w + 1];
    if (w < wave) lo_to += sums[2 * w], hi_to += sums[2 * w + 1];
  }
  // the bins before: x times 1 + 2^16 + 2^32 + 2^48 sums up the four counts in front of and in each
  lo_all *= 0x0001000100010001ull;
  hi_all *= 0x0001000100010001ull;
  lo_to += lo_all << 16;
  hi_to += (hi_all << 16) + (lo_all >> 48) * 0x0001000100010001ull;
  const int m0 = tid * words * 4;
  for (int i = 0; i < words; ++i)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const uint32_t bin = mine[i] >> (8 * e) & 255u;
      const int at = (int)((bin < 4 ? lo_to : hi_to) >> (16 * (bin & 3)) & 0xffffu);
      const uint64_t one = 1ull << (16 * (bin & 3));
      lo_to += bin < 4 ? one : 0;
      hi_to += bin >= 4 && bin < 8 ? one : 0;
      if (bin < 8) order[at] = make_int2(m0 + 4 * i + e, (int)bin < none ? (int)bin : -1);
    }
}

// 16 bytes per lane straight into LDS: lane l's land at `dst` + 16 l. (m0 is set in the block, which holds the wait state behind it.)
__device__ __forceinline__ void lane_to_lds(const void* p, uint32_t dst) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(dst), "v"(p) : "m0");
}
__device__ __forceinline__ void lds_reads_done() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }
template <int N>
__device__ __forceinline__ void vm_left() { asm volatile("s_waitcnt vmcnt(%0)" ::"i"(N) : "memory"); }

// t[z][m][r] of the rows of 16 T that name an adapter of this slot. The waves take steps of 64 k (a cache line of each row of x and A) in
// turns, each through a ring of NST steps in LDS of its own, and join in wave order. The operands' lanes lie row by row, 16 bytes of
// each: loaded so, a load takes 64 cycles of the address path (measured 15 bytes a cycle and CU, 42 us for 8192 rows of 4096, rank 64);
// into LDS eight lanes bring a row's line. Its eight chunks are moved by key_of(row) so that 16 rows' same chunk falls on different banks.
// RB: blocks of 16 ranks.
__device__ __forceinline__ int key_of(int row) { return row >> 1 & 7; }

template <int T, int RB, int W, int NST>
__global__ __launch_bounds__(64 * W) void k_lora_down(LoraArgs g) {
  constexpr int STAGE = 16 * (T + RB) * 128, RING = NST * STAGE, JOIN = W * 16 * (16 * T + 1) * 4, LDS = W * RING > JOIN ? W * RING : JOIN;
  static_assert(LDS <= 160 * 1024 && LDS >= 21 * 1024, "LDS");
  __shared__ __attribute__((aligned(1024))) char lds[LDS];
  const Lora& a = g.a;
  const int tid = threadIdx.x, lane = tid & 63, r16 = lane & 15, q4 = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  int at = blockIdx.x;
  if (g.order_out) {                                // the first of the workgroups
    if (at == 0) return order_few<W>(a, g.order_out, lds, wave, lane);
    --at;
  }
  const int z = at % g.splits;
  at /= g.splits;
  // slots last: the others' workgroups may have nothing to do
  const int tiles = (a.M + 16 * T - 1) / (16 * T), slot = at / tiles, m0 = tile_of(at % tiles, tiles) * 16 * T;
  const int2 place = place_of<16 * T>(g, m0, lane);
  const int mine = place.y;
  const int full = a.K >> 6, stride = g.splits * W, s0 = z * W + wave, n = full > s0 ? (full - s0 + stride - 1) / stride : 0;
  const char* ring = lds + wave * RING;
  const uint32_t ring0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)lds + wave * RING;

  auto body = [&](auto blocks, int ad, int rows, int count) __attribute__((always_inline)) {
    constexpr int MB = decltype(blocks)::value, LPS = 2 * (MB + RB);
    const int rank = rank_of(a, ad);
    const uint16_t *xa = a.a + ad * a.as;
    const uint16_t* from[LPS];                      // this lane's rows: x's (behind the last the first again, not written), A's
#pragma unroll
    for (int i = 0; i < LPS; ++i) {
      const int r = 8 * i + (lane >> 3), j = r - 16 * MB, ch = (lane & 7) ^ key_of(r);
      const int row = __shfl(rows, i < 2 * MB && r < count ? r : 0, 64);
      from[i] = (i < 2 * MB ? a.x + row * a.ldx : xa + (int64_t)min(j, a.R - 1) * a.K) + 8 * ch;
    }
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
    auto issue = [&](int at, int i) __attribute__((always_inline)) {
      const int64_t k = (int64_t)(s0 + i * stride) * 64;
#pragma unroll
      for (int l = 0; l < LPS; ++l) lane_to_lds(from[l] + k, ring0 + at * STAGE + l * 1024);
    };
    lds_reads_done();                               // (of the join before)
    vm_left<0>();
#pragma unroll
    for (int i = 0; i < NST - 1; ++i)
      if (i < n) issue(i, i);
    int at = 0;
    for (int i = 0; i < n; ++i) {
      lds_reads_done();
      if (i + NST - 1 < n) {
        issue(at == 0 ? NST - 1 : at - 1, i + NST - 1);
        vm_left<(NST - 1) * LPS>();
      } else {
        vm_left<0>();
      }
      const char* base = ring + at * STAGE;
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        auto frag = [&](int block) { return load16(base + (block * 16 + r16) * 128 + (((4 * u + q4) ^ key_of(r16)) << 4)); };
        uint4 xf[MB], af[RB];
#pragma unroll
        for (int mb = 0; mb < MB; ++mb) xf[mb] = frag(mb);
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) af[rb] = frag(MB + rb);
        multiply(xf, af);
      }
      at = at + 1 == NST ? 0 : at + 1;
    }
    if (a.K & 63 && s0 % stride == full % stride) {   // the last columns, no whole step
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const int k = full * 64 + 32 * u + 8 * q4;
        const bool in = k < a.K;                    // K is a multiple of 8
        uint4 xf[MB], af[RB];
#pragma unroll
        for (int mb = 0; mb < MB; ++mb) {
          const int j = mb * 16 + r16, row = __shfl(rows, j < count ? j : 0, 64);
          xf[mb] = in ? load16(a.x + row * a.ldx + k) : zeros();
        }
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) af[rb] = in ? load16(xa + (int64_t)min(rb * 16 + r16, a.R - 1) * a.K + k) : zeros();
        multiply(xf, af);
      }
    }
    const float scale = a.scales ? a.scales[ad] : 1.f;
    float(*part)[16][16 * T + 1] = reinterpret_cast<float(*)[16][16 * T + 1]>(lds);
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
        const int row = __shfl(rows, min(j, 63), 64);
        if (j < count && r < a.R) g.t[((int64_t)z * a.M + row) * a.R + r] = r < rank ? t * scale : 0.f;
      }
    }
    __syncthreads();
  };
  unsigned long long left = __ballot(mine >= 0);
  for (int j = 0; left; ++j) {
    const int ad = __builtin_amdgcn_readlane(mine, (int)__builtin_ctzll(left));
    const unsigned long long mask = __ballot(mine == ad);
    left &= ~mask;
    if (j % g.slots != slot) continue;
    const int rows = __shfl(place.x, nth_of(mask, lane), 64), count = __builtin_popcountll(mask);
    if (count > 16) body(std::integral_constant<int, T>(), ad, rows, count);
    else body(std::integral_constant<int, 1>(), ad, rows, count);
  }
}

// y of the rows of 64 that name an adapter of this slot (and in slot 0 those without one), g.run blocks of 64 outputs. The rows of one
// adapter go to the waves, 16 to each; the parts of t stay in registers. A block of B (64 rows, in memory as they lie) goes through
// registers into LDS, two blocks in turn, so that the next one's values and base are under way while one is computed. Product e's 16
// lanes of outputs are n = 64 nb + 4 l + e: a lane has four consecutive outputs of four rows, 16 lanes a row's 64. In LDS row 16 e + l holds that row of B, its chunks moved by at_of so that 16 rows' same chunk falls on
// different banks.
// HOW: kPast: results go past the caches; kParts: t is in several parts (few rows; without the code for that, results of many rows have
// a third wave on each SIMD: 8192 rows of 4096 x 4096, rank 64 70 us instead of 80). kFew, kFewParts: adapters of few rows are
// likely, the rank is 32 at most; they take up to 16 rows of an adapter without LDS, a block of outputs a wave (131 rows of 28 adapters in turn, 104 x
// 7680, rank 32 29 -> 20 us; 256 of 24, 4096 x 4096, rank 16 17 -> 14); at higher ranks that takes too many registers (64 rows of 24, rank 128 18 -> 25).
enum { kWhole, kPast, kParts, kFew, kFewParts };

template <bool F32, int RC, int HOW>
__global__ __launch_bounds__(256) void k_lora_up(LoraArgs g) {
  constexpr bool STREAM = HOW == kPast;
  constexpr int W = 4, PARTS = F32 ? 3 : 2, ROWS = 16 * W, PITCH = 64 * RC, CPR = 4 * RC, MINE = CPR / W;
  __shared__ __attribute__((aligned(16))) char lds[2][64 * PITCH];
  const Lora& a = g.a;
  const int tid = threadIdx.x, lane = tid & 63, r16 = lane & 15, q4 = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  // Workgroups are handed out to the eight XCDs in turn: a tile's outputs all go to one of them, so that its L2 cache sees whole
  // rows, not the same few columns (a few of its channels) of all rows. Slots last: the others' may have nothing to do.
  const int tiles = (a.M + ROWS - 1) / ROWS, xcds = g.xcds, each = (tiles + xcds - 1) / xcds, id = blockIdx.x;
  const int part = id / xcds % g.tiles_n, job = id / xcds / g.tiles_n, slot = job / each, tile = id % xcds * each + job % each;
  if (tile >= tiles) return;
  const int m0 = tile * ROWS, nb0 = part * g.run, nb1 = min(nb0 + g.run, (a.N + 63) / 64);
  auto at_of = [](int row, int ch) { return row * PITCH + ((ch ^ (RC == 1 ? row >> 2 & 3 : RC == 2 ? row >> 1 & 7 : row & 15)) << 4); };
  const int2 place = place_of<ROWS>(g, m0, lane);
  const int mine = place.y, lane_n = 4 * r16;

  // The rows whose bits are set in `mask`: of adapter ad (-1: none), or of none. FEW: 16 at most; the waves then take blocks of outputs
  // in turns, with B's values straight from memory.
  auto body = [&](auto few, int ad, unsigned long long mask) __attribute__((always_inline)) {
    constexpr bool FEW = decltype(few)::value;
    const int list = nth_of(mask, lane), count = __builtin_popcountll(mask), first = FEW ? 0 : wave * 16;
    const bool busy = first < count;
    const uint16_t* up = a.b + max(ad, 0) * a.bs;
    int m[4];                                       // rows of the results (behind the last: the first, not stored)
    bool with[4];                                   // do they have the adapter?
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int at = first + 4 * q4 + i, row = __shfl(list, at < count ? at : 0, 64);
      m[i] = __shfl(place.x, row, 64);
      with[i] = __shfl(mine, row, 64) >= 0;
    }
    // this lane's chunks of a block of B: read as far as R (what lies behind the rank is dropped below), the last row again behind N
    uint4 bw[MINE];
    auto load_b = [&](int nb) __attribute__((always_inline)) {
#pragma unroll
      for (int i = 0; i < MINE; ++i) {
        const int at = i * 64 * W + tid, row = at / CPR, ch = at % CPR;
        bw[i] = load16(up + (int64_t)min(nb * 64 + row, a.N - 1) * a.R + min(8 * ch, a.R - 8));
      }
    };
    auto keep_b = [&](char* to, int rank) __attribute__((always_inline)) {
#pragma unroll
      for (int i = 0; i < MINE; ++i) {
        const int at = i * 64 * W + tid, row = at / CPR, ch = at % CPR;
        *reinterpret_cast<uint4*>(to + at_of(16 * (row & 3) + (row >> 2), ch)) = first_of(bw[i], rank - 8 * ch);
      }
    };
    Base<F32, STREAM> base[4];
    auto load_base = [&](int nb) __attribute__((always_inline)) {
#pragma unroll
      for (int i = 0; i < 4; ++i) base[i].load(a, m[i], nb * 64 + lane_n);
    };
    // everything that is read goes under way before anything is waited for, the rank among it
    uint4 bv[FEW ? RC : 1][4];
    auto load_own = [&](int nb) __attribute__((always_inline)) {
#pragma unroll
      for (int rc = 0; rc < (FEW ? RC : 0); ++rc)
#pragma unroll
        for (int e = 0; e < 4; ++e)
          bv[rc][e] = load16(up + (int64_t)min(nb * 64 + 4 * r16 + e, a.N - 1) * a.R + min(rc * 32 + 8 * q4, a.R - 8));
    };
    if constexpr (FEW) {
      if (nb0 + wave >= nb1) return;
      if (ad >= 0) load_own(nb0 + wave);
      load_base(nb0 + wave);
    } else {
      if (ad >= 0) load_b(nb0);
      if (busy) load_base(nb0);
    }
    const int at = __shfl(list, first + r16 < count ? first + r16 : 0, 64), row = __shfl(place.x, at, 64);
    const bool has = __shfl(mine, at, 64) >= 0;
    f32x4 tv[RC][2];
    auto load_t = [&](int z, int rc, int i) __attribute__((always_inline)) {
      return *reinterpret_cast<const f32x4*>(g.t + ((int64_t)z * a.M + row) * a.R + min(rc * 32 + 8 * q4, a.R - 8) + 4 * i);
    };
#pragma unroll
    for (int rc = 0; rc < RC; ++rc)
#pragma unroll
      for (int i = 0; i < 2; ++i) tv[rc][i] = ad >= 0 && busy ? load_t(0, rc, i) : f32x4{0, 0, 0, 0};
    const int rank = ad < 0 ? 0 : rank_of(a, ad);
    uint4 tf[RC][PARTS];
    if (rank && busy) {
      // the parts in their order, a few asked for at once (one behind the other, 64 rows of 24 adapters, 4096 x 4096, rank 16 / 128 took
      // 11.7 / 24.8 us, so 10.7 / 18.0)
      if constexpr (HOW == kParts || HOW == kFewParts) {
        auto add = [&](auto count, int z0) __attribute__((always_inline)) {
          constexpr int Z = decltype(count)::value;
          f32x4 more[Z][RC][2];
#pragma unroll
          for (int u = 0; u < Z; ++u)
#pragma unroll
            for (int rc = 0; rc < RC; ++rc)
#pragma unroll
              for (int i = 0; i < 2; ++i) more[u][rc][i] = load_t(z0 + u, rc, i);
#pragma unroll
          for (int u = 0; u < Z; ++u)
#pragma unroll
            for (int rc = 0; rc < RC; ++rc)
#pragma unroll
              for (int i = 0; i < 2; ++i) tv[rc][i] += more[u][rc][i];
        };
        constexpr int Z = RC == 1 ? 7 : RC == 2 ? 3 : 2;
        int z = 1;
        for (; z + Z <= g.splits; z += Z) add(std::integral_constant<int, Z>(), z);
        for (; z < g.splits; ++z) add(std::integral_constant<int, 1>(), z);
      }
#pragma unroll
      for (int rc = 0; rc < RC; ++rc) {
        const int held = has ? rank - rc * 32 - 8 * q4 : 0;                             // of this lane's eight ranks
        float t[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) t[i] = i < held ? tv[rc][i / 4][i % 4] : 0.f;
#pragma unroll
        for (int p = 0; p < PARTS; ++p) {
          uint32_t w[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            w[i] = f2bf2(t[2 * i], t[2 * i + 1]);
            t[2 * i] = rest_of(t[2 * i], (uint16_t)w[i]);
            t[2 * i + 1] = rest_of(t[2 * i + 1], (uint16_t)(w[i] >> 16));
          }
          tf[rc][p] = make_uint4(w[0], w[1], w[2], w[3]);
        }
      }
    }
    // results of a block, of four rows
    auto finish = [&](int nb, int next, const f32x4 (&acc)[4]) __attribute__((always_inline)) {
      // lane holds its outputs of rows 4 q4 + i
      f32x4 v[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        v[i] = base[i].values();
        if (with[i]) v[i] += f32x4{acc[0][i], acc[1][i], acc[2][i], acc[3][i]};
      }
      if (next < nb1) load_base(next);
      activate(v, a.act);
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (first + 4 * q4 + i < count) store<F32, STREAM>(a, m[i], nb * 64 + lane_n, v[i]);
    };
    if constexpr (FEW) {
      for (int nb = nb0 + wave; nb < nb1; nb += W) {
        f32x4 acc[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[e] = f32x4{0, 0, 0, 0};
#pragma unroll
        for (int rc = 0; rc < RC; ++rc)
          if (rc * 32 < rank) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const bf16x8 bf = as_bf16x8(first_of(bv[rc][e], rank - rc * 32 - 8 * q4));
#pragma unroll
              for (int p = 0; p < PARTS; ++p) acc[e] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(tf[rc][p]), bf, acc[e], 0, 0, 0);
            }
          }
        if (rank && nb + W < nb1) load_own(nb + W);
        finish(nb, nb + W, acc);
      }
      return;
    }
    __syncthreads();                                // (the last adapter's block has been read)
    if (rank) keep_b(lds[0], rank);
    __syncthreads();
    for (int nb = nb0; nb < nb1; ++nb) {
      const char* b = lds[(nb - nb0) & 1];
      if (rank && nb + 1 < nb1) load_b(nb + 1);
      if (busy) {
        f32x4 acc[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[e] = f32x4{0, 0, 0, 0};
#pragma unroll
        for (int rc = 0; rc < RC; ++rc)
          if (rc * 32 < rank) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const bf16x8 bf = as_bf16x8(load16(b + at_of(16 * e + r16, 4 * rc + q4)));
#pragma unroll
              for (int p = 0; p < PARTS; ++p) acc[e] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(tf[rc][p]), bf, acc[e], 0, 0, 0);
            }
          }
        finish(nb, nb + 1, acc);
      }
      if (rank && nb + 1 < nb1) {
        keep_b(lds[(nb + 1 - nb0) & 1], rank);
        __syncthreads();
      }
    }
  };
  unsigned long long left = __ballot(mine >= 0);
  // rows without an adapter go with the first adapter's, or by themselves
  const unsigned long long none = __ballot(m0 + lane < a.M) & ~left;
  int j = 0;
  do {
    const int ad = left ? __builtin_amdgcn_readlane(mine, (int)__builtin_ctzll(left)) : -1;
    const unsigned long long mask = __ballot(mine == ad) & left;
    left &= ~mask;
    if (j++ % g.slots == slot) {
      const unsigned long long rows = j > 1 ? mask : mask | none;
      if constexpr (HOW == kFew || HOW == kFewParts) {
        if (__builtin_popcountll(rows) <= 16) {
          body(std::true_type(), ad, rows);
          continue;
        }
      }
      body(std::false_type(), ad, rows);
    }
  } while (left);
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
  const int mine = row ? adapter_of(a, m) : -1;
  const uint16_t* x = a.x + (row ? m : m0) * a.ldx;

  f32x4 acc[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) acc[e] = f32x4{0, 0, 0, 0};
  uint32_t left = (uint32_t)__ballot(mine >= 0) & 0xffffu;
  while (left) {
    const int ad = __builtin_amdgcn_readlane(mine, __builtin_ctz(left));
    left &= ~(uint32_t)__ballot(mine == ad);
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
        const int n = n0 + 4 * r16 + e;
        const uint4 bf = n < a.N && r < rank ? first_of(load16(up + (int64_t)n * a.R + r), rank - r) : zeros();
#pragma unroll
        for (int p = 0; p < PARTS; ++p) y[e] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(tf[p], as_bf16x8(bf), y[e], 0, 0, 0);
      }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (__shfl(mine, 4 * q4 + i, 64) != ad) continue;
#pragma unroll
      for (int e = 0; e < 4; ++e) acc[e][i] = y[e][i];
    }
  }
  // lane holds its outputs of rows 4 q4 + i
  f32x4 v[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    Base<F32, false> base;
    base.load(a, min(m0 + 4 * q4 + i, a.M - 1), n0 + 4 * r16);
    v[i] = base.values() + f32x4{acc[0][i], acc[1][i], acc[2][i], acc[3][i]};
  }
  activate(v, a.act);
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (m0 + 4 * q4 + i < a.M) store<F32, false>(a, m0 + 4 * q4 + i, n0 + 4 * r16, v[i]);
}

unsigned up_grid(const LoraArgs& g) {
  const int tiles = (g.a.M + 63) / 64;
  return (unsigned)((tiles + g.xcds - 1) / g.xcds * g.xcds) * g.slots * g.tiles_n;
}

template <bool F32, int HOW>
hipError_t up(const LoraArgs& g, hipStream_t s) {
  const unsigned wgs = up_grid(g);
  const int rc = (g.a.R + 31) / 32;
  return launch(rc == 1 ? k_lora_up<F32, 1, HOW> : rc == 2 ? k_lora_up<F32, 2, HOW> : k_lora_up<F32, 4, HOW>, dim3(wgs), dim3(256), 0, s, g);
}

// All rows of a call, or a part of them. p: the plan of a whole part, for the last one too, so that every row's sums are added in the same order.
hipError_t rows_of(const Lora& a, const LoraPlan& p, const Split& sp, hipStream_t s) {
  LoraArgs g{};
  g.a = a;
  g.t = sp.partials;
  g.tiles_n = (int)(((int64_t)a.N + 255) / 256);
  if (p.splits == 0)
    return launch(a.f32 ? k_lora<true> : k_lora<false>, dim3((unsigned)((a.M + 15) / 16 * g.tiles_n)), dim3(64 * kWaves), 0, s, g);
  g.splits = p.splits;
  int2* const order = reinterpret_cast<int2*>(g.t + (int64_t)p.splits * a.M * a.R);       // (R is even: at 8 bytes)
  if (p.order == 1) {
    g.order = order;
    const hipError_t e = launch(k_lora_order, dim3(1), dim3(1024), 0, s, g);
    if (e != hipSuccess) return e;
  }
  g.order_out = p.order == 2 ? order : nullptr;
  g.slots = p.down_slots;
  const unsigned tiles = p.tall ? (a.M + 63) / 64 : (a.M + 31) / 32;
  const int rb = (a.R + 15) / 16;
  const unsigned down = tiles * g.slots * g.splits + (p.order == 2);
  const hipError_t e = rb == 1   ? launch(k_lora_down<2, 1, 4, 2>, dim3(down), dim3(256), 0, s, g)
                       : rb == 2 ? launch(k_lora_down<2, 2, 4, 2>, dim3(down), dim3(256), 0, s, g)
                       : p.tall  ? launch(k_lora_down<4, 4, 2, 2>, dim3(down), dim3(128), 0, s, g)
                       : rb <= 4 ? launch(k_lora_down<2, 4, 3, 2>, dim3(down), dim3(192), 0, s, g)
                                 : launch(k_lora_down<2, 8, 4, 1>, dim3(down), dim3(256), 0, s, g);
  if (e != hipSuccess) return e;
  if (p.order) g.order = order;
  g.slots = p.up_slots;
  g.run = p.run;
  g.xcds = a.M <= 7 * 64 ? 1 : 8;                   // fewer than eight tiles: one
  g.tiles_n = (int)((((int64_t)a.N + 63) / 64 + g.run - 1) / g.run);
  // A result of 16 MiB or more goes past the caches, as its base comes, where rows are whole lines of 128 bytes (8192 rows of 4096 x
  // 4096, rank 64: 69 us instead of 78; 8191 rows of 4096 x 4099, whose lines are written in two parts, 104 so and 85 through the caches).
  const int64_t item = a.f32 ? 4 : 2;
  const bool lines = (((uintptr_t)a.y | (uintptr_t)a.base | (uintptr_t)(a.ldy * item) | (uintptr_t)(a.ldbase * item)) & 127) == 0;
  if (a.R <= 32 && !p.order && (a.adapters >= 4 || a.M <= 16)) {        // a tile's 64 rows are of so many, or it has no more
    const auto few = g.splits == 1 ? (a.f32 ? k_lora_up<true, 1, kFew> : k_lora_up<false, 1, kFew>)
                                   : (a.f32 ? k_lora_up<true, 1, kFewParts> : k_lora_up<false, 1, kFewParts>);
    return launch(few, dim3(up_grid(g)), dim3(256), 0, s, g);
  }
  if (g.splits > 1) return a.f32 ? up<true, kParts>(g, s) : up<false, kParts>(g, s);
  if (lines && (int64_t)a.M * a.N * item >= 16 << 20) return a.f32 ? up<true, kPast>(g, s) : up<false, kPast>(g, s);
  return a.f32 ? up<true, kWhole>(g, s) : up<false, kWhole>(g, s);
}

}  // namespace

hipError_t lora(const Lora& a, const Split& sp, hipStream_t s) {
  if (!a.x || !a.a || !a.b || !a.adapter || !a.y || a.M < 1 || a.N < 1 || a.K < 8 || a.K % 8 || a.R < 8 || a.R % 8 || a.R > kLoraRank ||
      a.adapters < 1)
    return hipErrorInvalidValue;
  if (((int64_t)a.M + 15) / 16 * (((int64_t)a.N + 255) / 256) >= 1 << 24) return hipErrorInvalidValue;
  const uint64_t scratch = sp.partials ? sp.partial_bytes : 0;
  const int64_t rows = lora_rows(a.M, a.N, a.K, a.R, a.adapters, scratch), item = a.f32 ? 4 : 2;
  const LoraPlan plan = lora_plan(rows, a.N, a.K, a.R, a.adapters, scratch);
  for (int64_t m0 = 0; m0 < a.M; m0 += rows) {
    Lora part = a;
    part.M = (int)std::min<int64_t>(rows, a.M - m0);
    part.x += m0 * a.ldx;
    part.adapter += m0;
    if (a.base) part.base = static_cast<const char*>(a.base) + m0 * a.ldbase * item;
    part.y = static_cast<char*>(a.y) + m0 * a.ldy * item;
    const hipError_t e = rows_of(part, plan, sp, s);
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace k
}  // namespace tp
