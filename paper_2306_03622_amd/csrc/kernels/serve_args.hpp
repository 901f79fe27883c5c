// What the serving operators' kernels share: a sequence's lengths. (No model's graph runs them, so their argument blocks name no pointers to
// the launch log, as those of gemm_args.hpp do.)
#pragma once
#include "common.hpp"

namespace tp {
namespace k {

// New and held tokens of a sequence.
struct Lens {
  int qn, kn;
};
__device__ __forceinline__ Lens lens_of(const Pages& p, int b) {
  Lens l;
  l.qn = p.q_lens ? min(max(p.q_lens[b], 0), p.q_len) : p.q_len;
  l.kn = min(max(p.kv_lens[b], 0), 1 << 30);
  return l;
}

}  // namespace k
}  // namespace tp
