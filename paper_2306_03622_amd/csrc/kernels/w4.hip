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
#include "gemm_tile.hpp"
#include "w4_plan.hpp"

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

// The two constants of the unpacking, in registers that the compiler knows nothing about: with literals it takes two
// instructions for (x & mask) | one, a third more of the tiled kernel's. (The instruction itself is left to the compiler, which
// keeps its distance from matrix instructions that still read or write its registers; it does not for one in assembly.)
struct W4Unpack {
  uint32_t mask = 0x00780078u, one = 0x41804180u;
  __device__ __forceinline__ W4Unpack() {
    asm("" : "+s"(mask));
    asm("" : "+v"(one));
  }
  // eight codes as bf16 16 + c, column order
  __device__ __forceinline__ bf16x8 operator()(uint32_t w) const {
    return as_bf16x8(make_uint4(((w << 3) & mask) | one, ((w >> 1) & mask) | one, ((w >> 5) & mask) | one,
                                ((w >> 9) & mask) | one));
  }
};

// the constant operand -24 in every place
__device__ __forceinline__ bf16x8 w4_surplus() {
  return as_bf16x8(make_uint4(0xC1C0C1C0u, 0xC1C0C1C0u, 0xC1C0C1C0u, 0xC1C0C1C0u));
}

// ReLU of what is not a number is not one either (act_apply gives 0): a row that an infinite or NaN input has spoilt shows it.
__device__ __forceinline__ float w4_act(float v, int act) {
  if (act == ACT_RELU) return v <= 0.f ? 0.f : v;
  return act_apply(v, act);
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
    for (int e = 0; e < 4; ++e) v[e] = w4_act(v[e], a.act);
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
    t = w4_act(t, a.act);
    if (a.y_f32) static_cast<float*>(a.y)[at + e] = t;
    else static_cast<uint16_t*>(a.y)[at + e] = f2bf(t);
  }
}

// One k-block: acc[i][t] += scales of weight block i times its codes' products with activation block t. xf holds the
// activations' four 32-column steps, wv the blocks' codes, sv their scales, four rows a lane and group.
template <int MB, int NB, int GP>
__device__ __forceinline__ void w4_block(const uint4 (&xf)[MB][4], const uint4 (&wv)[NB], const uint2 (&sv)[NB][GP],
                                         f32x4 (&acc)[NB][MB]) {
  constexpr int SPG = 4 / GP;             // 32-column steps per group
  const bf16x8 surplus = w4_surplus();
  const W4Unpack unpack;
#pragma unroll
  for (int p = 0; p < GP; ++p) {
    f32x4 xs[MB];
#pragma unroll
    for (int t = 0; t < MB; ++t) xs[t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int j = p * SPG; j < (p + 1) * SPG; ++j)
#pragma unroll
      for (int t = 0; t < MB; ++t)
        xs[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(surplus, as_bf16x8(xf[t][j]), xs[t], 0, 0, 0);
#pragma unroll
    for (int i = 0; i < NB; ++i) {
      const uint32_t w4[4] = {wv[i].x, wv[i].y, wv[i].z, wv[i].w};
      f32x4 sum[MB];
#pragma unroll
      for (int t = 0; t < MB; ++t) sum[t] = xs[t];
#pragma unroll
      for (int j = p * SPG; j < (p + 1) * SPG; ++j) {
        const bf16x8 wf = unpack(w4[j]);
#pragma unroll
        for (int t = 0; t < MB; ++t)
          sum[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wf, as_bf16x8(xf[t][j]), sum[t], 0, 0, 0);
      }
      const float s4[4] = {bf2f(sv[i][p].x & 0xffff), bf2f(sv[i][p].x >> 16), bf2f(sv[i][p].y & 0xffff), bf2f(sv[i][p].y >> 16)};
#pragma unroll
      for (int t = 0; t < MB; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[i][t][e] = fmaf(s4[e], sum[t][e], acc[i][t][e]);
    }
  }
}

// Few rows: a workgroup owns 16 NB weight rows and 16 MT activation rows, its NW waves a contiguous run of k-blocks
// each; they add up through LDS in wave order. One 16-byte load per lane brings a whole 1 KB block of weights. A wave
// keeps U k-blocks in flight: block u's registers take the block U further on as soon as they are multiplied. Loads beyond
// a wave's run, the rows or the columns go out of their buffer's bounds, which reads zeros and moves nothing, so nothing
// in the loop is conditional.
//
// Bound by the weights' way from HBM where there are many (1 x 32768 x 8192, 138 MB: 30 to 33 us, 4.2 to 4.6 TB/s, where a read
// alone reaches 6.1), else by the chain of a launch, the loads' round trips and a reduction: 1 x 768 x 768 3.0 us (an empty
// launch takes about as much); 8 x 4096 x 4096 5.9 us, eight k-blocks a wave, two in flight: four turns, matrix instructions in 8% of the
// time and vector ones in 15%; 100 x 1000 x 2048 5.9, both k-blocks of a wave in flight. Waves split the columns, not the rows, so that the
// loads of a few hundred workgroups cover the latency.
template <int MT, int NB, int NW, int GP, int U>
__global__ __launch_bounds__(NW * 64) void k_w4_rows(W4Args g) {
  const LinearW4& a = g.a;
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int r = lane & 15, q = lane >> 4;
  const int nb0 = blockIdx.x * NB, m0 = blockIdx.y * (16 * MT);
  const int nbs = min(((a.N + 15) >> 4) - nb0, NB), rows = min(a.M - m0, 16 * MT);
  const __amdgpu_buffer_rsrc_t rx = buffer_of(a.x + (int64_t)m0 * a.ldx, (uint32_t)(((rows - 1) * a.ldx + a.K) * 2));
  const __amdgpu_buffer_rsrc_t rw = buffer_of(a.wq + (int64_t)nb0 * g.kb * 1024, (uint32_t)(nbs * g.kb) * 1024u);
  const __amdgpu_buffer_rsrc_t rs = buffer_of(a.scales + (int64_t)nb0 * g.groups * 16, (uint32_t)(nbs * g.groups) * 32u);
  uint32_t offx[MT], offw[NB], offs[NB];
#pragma unroll
  for (int t = 0; t < MT; ++t) offx[t] = 16 * t + r < rows ? (uint32_t)(16 * t + r) * (uint32_t)(a.ldx * 2) + q * 16 : kOffNone;
#pragma unroll
  for (int b = 0; b < NB; ++b) {
    offw[b] = b < nbs ? (uint32_t)(b * g.kb) * 1024u + lane * 16 : kOffNone;
    offs[b] = b < nbs ? (uint32_t)(b * g.groups) * 32u + q * 8 : kOffNone;
  }
  const int per = (g.kb + NW - 1) / NW, kb0 = wave * per, kb_end = min(g.kb, kb0 + per);
  uint4 wv[U][NB], xv[U][MT][4];
  uint2 sv[U][NB][GP];
  auto load = [&](int u, int kb) __attribute__((always_inline)) {
    const bool in = kb < kb_end;
#pragma unroll
    for (int b = 0; b < NB; ++b) {
      wv[u][b] = buffer_load16(rw, in ? offw[b] + (uint32_t)kb * 1024u : kOffNone);
#pragma unroll
      for (int p = 0; p < GP; ++p)
        sv[u][b][p] = __builtin_bit_cast(
            uint2, __builtin_amdgcn_raw_buffer_load_b64(rs, in ? offs[b] + (uint32_t)(kb * GP + p) * 32u : kOffNone, 0, 0));
    }
#pragma unroll
    for (int t = 0; t < MT; ++t)
#pragma unroll
      for (int j = 0; j < 4; ++j)
        xv[u][t][j] = buffer_load16(rx, in && kb * 128 + 32 * j < a.K ? offx[t] + (uint32_t)(kb * 256 + 64 * j) : kOffNone);
  };
  f32x4 acc[NB][MT];
#pragma unroll
  for (int b = 0; b < NB; ++b)
#pragma unroll
    for (int t = 0; t < MT; ++t) acc[b][t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int u = 0; u < U; ++u) load(u, kb0 + u);
  for (int kb = kb0; kb < kb_end; kb += U) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      w4_block<MT, NB, GP>(xv[u], wv[u], sv[u], acc);
      load(u, kb + u + U);
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

// Many rows: a BN x BM output tile. KS sets of WGN x WGM waves (16 NB x 16 MB outputs each) take 128-column blocks by
// turns, set ks the blocks ks, ks + KS, .., and add up at the end, in the order of the sets: with few workgroups a
// wave's block is a chain of dependent LDS reads, multiplications and a barrier, which other sets' blocks fill.
//
// A ring of NST stages (KS blocks each) in LDS filled by loads that go straight there (lds_load16, as in gemm_tile.hpp):
// the activations as rows of 256 bytes whose 16-byte chunk c lies at position c ^ row % 16 (the 16 rows read together
// fall on different banks), the weights as the 1 KB blocks they are, the blocks' scales behind them. Every wave issues
// the same LPS loads a stage, so one count tells when a stage has landed. A block's activation fragments stay in registers
// while the weight blocks pass: one is unpacked once, multiplied with all MB fragments, and its scale applied to the
// finished group.
//
// Bound, for the largest tiles, by matrix and vector instructions that hardly overlap: 8192 x 4096 x 4096 in groups of 128
// takes 302 us, 0.91 PFLOP/s (a plain bf16 product of that size by the library 214 us). Beside 80 matrix instructions (16 cycles each) a
// wave issues about 275 vector ones (4 each) a stage; the matrix pipes are busy 47% of the time, the vector ones 41%, and the two waves of a
// SIMD leave the same barrier together. Neither waves of 32 rows x 128 outputs (11% slower), nor activation sums shared between
// waves (2%), nor fragments read half a stage ahead gained anything. Mid sizes are chains of few stages: 1024 x 2304 x 768 12.1 us, six
// stages on 576 workgroups, of which 64 CUs hold three and the others two.
template <int BN, int BM, int WGN, int WGM, int KS, int NST, int GP>
struct W4Tile {
  static constexpr int NW = WGN * WGM, NB = BN / WGN / 16, MB = BM / WGM / 16;
  static constexpr int TX = BM / 4 / NW, TW = BN / 16 / NW, LPS = TX + TW + 1;
  static constexpr int ITEMS = BN / 8 * GP, SPARTS = ITEMS > 64 ? ITEMS / 64 : 1;   // 16-byte pieces of scales
  static constexpr int XB = BM * 256, WB = BN * 64, BLOCK = XB + WB + SPARTS * 1024, SBYTES = KS * BLOCK;
  static constexpr size_t join = (size_t)(KS - 1) * NW * 64 * NB * MB * 16;
  static constexpr size_t ring = (size_t)NST * SBYTES, lds = ring > join ? ring : join;
  static_assert(TX >= 1 && TW >= 1 && BM % (4 * NW) == 0 && BN % (16 * NW) == 0 && NW % SPARTS == 0 && lds <= 160 * 1024,
                "tile shape");
};

template <int BN, int BM, int WGN, int WGM, int KS, int NST, int GP, int MINW>
__global__ __launch_bounds__(64 * WGN * WGM * KS, MINW) void k_w4_tile(W4Args g, int tn, int tm) {
  typedef W4Tile<BN, BM, WGN, WGM, KS, NST, GP> T;
  constexpr int NB = T::NB, MB = T::MB;
  __shared__ __attribute__((aligned(1024))) char lds[T::lds];
  const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)lds;
  const LinearW4& a = g.a;
  const int tid = threadIdx.x, lane = tid & 63;
  const int all = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int ks = all / T::NW, wave = all % T::NW, wn = wave % WGN, wm = wave / WGN;
  const int r = lane & 15, q = lane >> 4;
  const TileAt at = tile_at<false>(blockIdx.x, gridDim.x, tn, tm, 1);
  const int nb0 = at.tx * (BN / 16), m0 = at.ty * BM;
  const int nbs = ((a.N + 15) >> 4) - nb0, rows = a.M - m0;            // blocks and rows from here to the end
  const int n = (g.kb + KS - 1) / KS;                                  // stages

  const __amdgpu_buffer_rsrc_t rx = buffer_of(a.x + (int64_t)m0 * a.ldx, (uint32_t)((min(rows, BM) - 1) * a.ldx * 2 + a.K * 2));
  const __amdgpu_buffer_rsrc_t rw = buffer_of(a.wq + (int64_t)nb0 * g.kb * 1024, (uint32_t)min(nbs, BN / 16) * g.kb * 1024u);
  const __amdgpu_buffer_rsrc_t rs = buffer_of(a.scales + (int64_t)nb0 * g.groups * 16, (uint32_t)min(nbs, BN / 16) * g.groups * 32u);
  uint32_t offx[T::TX], offw[T::TW], offs;
  int chx[T::TX];
#pragma unroll
  for (int t = 0; t < T::TX; ++t) {
    const int row = (wave * T::TX + t) * 4 + (lane >> 4);
    chx[t] = ((lane & 15) ^ (row & 15)) * 8;
    offx[t] = row < rows ? (uint32_t)(row * (uint32_t)a.ldx + chx[t]) * 2 : kOffNone;
  }
#pragma unroll
  for (int t = 0; t < T::TW; ++t) {
    const int nb = wave * T::TW + t;
    offw[t] = nb < nbs ? (uint32_t)(nb * g.kb) * 1024u + lane * 16 : kOffNone;
  }
  {
    const int item = (wave % T::SPARTS) * 64 + lane, nb = item / (2 * GP);
    offs = item < T::ITEMS && nb < nbs ? (uint32_t)(nb * g.groups) * 32u + (item % (2 * GP)) * 16 : kOffNone;
  }
  // this set's block of stage st; one beyond the last reads zeros
  auto issue = [&](int slot, int st) __attribute__((always_inline)) {
    const int kb = st * KS + ks;
    const uint32_t dst = lds0 + slot * T::SBYTES + ks * T::BLOCK;
    const int left = a.K - kb * 128;              // columns from here to the end
    if (left >= 128) {
#pragma unroll
      for (int t = 0; t < T::TX; ++t) lds_load16<false>(rx, dst + (wave * T::TX + t) * 1024, offx[t], kb * 256);
#pragma unroll
      for (int t = 0; t < T::TW; ++t) lds_load16<false>(rw, dst + T::XB + (wave * T::TW + t) * 1024, offw[t], kb * 1024);
      lds_load16<false>(rs, dst + T::XB + T::WB + (wave % T::SPARTS) * 1024, offs, kb * GP * 32);
      return;
    }
    const bool in = left > 0;
#pragma unroll
    for (int t = 0; t < T::TX; ++t)
      lds_load16<false>(rx, dst + (wave * T::TX + t) * 1024, chx[t] < left ? offx[t] : kOffNone, in ? kb * 256 : 0);
#pragma unroll
    for (int t = 0; t < T::TW; ++t)
      lds_load16<false>(rw, dst + T::XB + (wave * T::TW + t) * 1024, in ? offw[t] : kOffNone, in ? kb * 1024 : 0);
    lds_load16<false>(rs, dst + T::XB + T::WB + (wave % T::SPARTS) * 1024, in ? offs : kOffNone, in ? kb * GP * 32 : 0);
  };

  f32x4 acc[NB][MB];
#pragma unroll
  for (int i = 0; i < NB; ++i)
#pragma unroll
    for (int j = 0; j < MB; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  uint32_t rdx[4];                                // byte offsets of this lane's fragments of a 16-row block
#pragma unroll
  for (int j = 0; j < 4; ++j) rdx[j] = (wm * MB * 16 + r) * 256 + (((4 * j + q) ^ r) << 4);

#pragma unroll
  for (int i = 0; i < NST - 1; ++i)
    if (i < n) issue(i, i);
  int slot = 0;
  for (int st = 0; st < n; ++st) {
    // stage st has landed for every wave, and the slot of stage st - 1 is free
    if (st + NST - 2 < n) lds_wait_barrier<(NST - 2) * T::LPS>();
    else lds_wait_barrier<0>();
    if (st + NST - 1 < n) issue(slot == 0 ? NST - 1 : slot - 1, st + NST - 1);
    const char* base = lds + slot * T::SBYTES + ks * T::BLOCK;
    uint4 xf[MB][4], wv[NB];
    uint2 sv[NB][GP];
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
      for (int t = 0; t < MB; ++t) xf[t][j] = *reinterpret_cast<const uint4*>(base + rdx[j] + t * 4096);
#pragma unroll
    for (int i = 0; i < NB; ++i) {
      wv[i] = *reinterpret_cast<const uint4*>(base + T::XB + (wn * NB + i) * 1024 + lane * 16);
#pragma unroll
      for (int p = 0; p < GP; ++p)
        sv[i][p] = *reinterpret_cast<const uint2*>(base + T::XB + T::WB + ((wn * NB + i) * GP + p) * 32 + q * 8);
    }
    w4_block<MB, NB, GP>(xf, wv, sv, acc);
    slot = slot + 1 == NST ? 0 : slot + 1;
  }
  if constexpr (KS > 1) {
    f32x4* area = reinterpret_cast<f32x4*>(lds) + (size_t)wave * 64 * NB * MB + lane;
    constexpr int set = T::NW * 64 * NB * MB;
    __syncthreads();
    if (ks > 0) {
#pragma unroll
      for (int i = 0; i < NB; ++i)
#pragma unroll
        for (int t = 0; t < MB; ++t) area[(ks - 1) * set + (i * MB + t) * 64] = acc[i][t];
    }
    __syncthreads();
    if (ks > 0) return;
#pragma unroll
    for (int x = 0; x < KS - 1; ++x)
#pragma unroll
      for (int i = 0; i < NB; ++i)
#pragma unroll
        for (int t = 0; t < MB; ++t) acc[i][t] += area[x * set + (i * MB + t) * 64];
  }
#pragma unroll
  for (int t = 0; t < MB; ++t)
#pragma unroll
    for (int i = 0; i < NB; ++i) w4_store(g, m0 + (wm * MB + t) * 16 + r, (nb0 + wn * NB + i) * 16 + 4 * q, acc[i][t]);
}

template <int BN, int BM, int WGN, int WGM, int KS, int NST, int MINW>
hipError_t go_tile(const W4Args& g, hipStream_t s) {
  constexpr int threads = 64 * WGN * WGM * KS;
  const int tn = (g.a.N + BN - 1) / BN, tm = (g.a.M + BM - 1) / BM;
  const dim3 grid((unsigned)tn * tm), block(threads);
  switch (g.a.group) {
    case 128: return launch((k_w4_tile<BN, BM, WGN, WGM, KS, NST, 1, MINW>), grid, block, 0, s, g, tn, tm);
    case 64: return launch((k_w4_tile<BN, BM, WGN, WGM, KS, NST, 2, MINW>), grid, block, 0, s, g, tn, tm);
    default: return launch((k_w4_tile<BN, BM, WGN, WGM, KS, NST, 4, MINW>), grid, block, 0, s, g, tn, tm);
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

hipError_t linear_w4(const LinearW4& a, hipStream_t s) {
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
  // 32-bit offsets of the rows a workgroup owns
  if (a.ldx >= (1 << 30) / 128) return hipErrorInvalidValue;
  switch (w4_plan(a.M, a.N, a.K, a.group)) {     // rows: MT, NB, waves, k-blocks in flight; tiles: waves n x m, sets, ring, waves per SIMD
    case W4_ROWS16: return go_rows<1, 1, 4, 2>(g, s);
    case W4_ROWS32: return go_rows<1, 2, 8, 2>(g, s);
    case W4_ROWS64: return go_rows<1, 4, 8, 1>(g, s);
    case W4_TILE32X32: return go_tile<32, 32, 2, 1, 4, 3, 2>(g, s);
    case W4_TILE64X32: return go_tile<64, 32, 4, 1, 2, 3, 2>(g, s);
    case W4_TILE64X32_DEEP: return go_tile<64, 32, 4, 1, 4, 2, 4>(g, s);
    case W4_TILE64X64: return go_tile<64, 64, 2, 2, 1, 2, 2>(g, s);
    case W4_TILE128X64: return go_tile<128, 64, 4, 2, 1, 2, 2>(g, s);
    case W4_TILE128X64_WIDE: return go_tile<128, 64, 4, 1, 1, 2, 2>(g, s);
    case W4_TILE256X128: return go_tile<256, 128, 4, 2, 1, 3, 2>(g, s);
    default: return hipErrorInvalidValue;        // no variant's grid holds so many outputs
  }
}

}  // namespace k
}  // namespace tp
