// What the serving operators' kernels share: the pointers of their argument blocks and a sequence's lengths.
#pragma once
#include "common.hpp"

namespace tp {
namespace k {

inline void add_ptrs(std::vector<uint32_t>& v, uint32_t at, std::initializer_list<size_t> fields) {
  for (size_t o : fields) v.push_back(at + (uint32_t)o);
}

template <>
struct PtrFields<CacheRows> {
  static void add(std::vector<uint32_t>& v, uint32_t at) {
    add_ptrs(v, at, {offsetof(CacheRows, c) + offsetof(Cache, k), offsetof(CacheRows, c) + offsetof(Cache, v),
                     offsetof(CacheRows, c) + offsetof(Cache, exps), offsetof(CacheRows, p) + offsetof(Pages, table),
                     offsetof(CacheRows, p) + offsetof(Pages, q_lens), offsetof(CacheRows, p) + offsetof(Pages, kv_lens),
                     offsetof(CacheRows, k), offsetof(CacheRows, v)});
  }
};

template <>
struct PtrFields<Lora> {
  static void add(std::vector<uint32_t>& v, uint32_t at) {
    add_ptrs(v, at, {offsetof(Lora, x), offsetof(Lora, a), offsetof(Lora, b), offsetof(Lora, adapter), offsetof(Lora, ranks),
                     offsetof(Lora, scales), offsetof(Lora, base), offsetof(Lora, y)});
  }
};

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
