// The serving operators' C entry points (torpor_serve.h): argument checks, the device of the stream, the launch.
#include "torpor_serve.h"

#include <algorithm>
#include <cmath>

#include "../kernels/kernels.hpp"
#include "ops_common.hpp"

using namespace tp;

namespace {

// The pool, with strides in bytes; those of a dimension of one entry are not used. An error's text, or null.
const char* cache_of(const tps_cache& c, k::Cache* to) {
  if (c.dtype != TP_BF16 && c.dtype != TPS_E4M3) return "the cache's dtype must be TP_BF16 or TPS_E4M3";
  if (c.reserved != 0) return "reserved must be 0";
  if (c.head_dim != 64 && c.head_dim != 128) return "head_dim must be 64 or 128";
  if (c.pages < 1 || c.kv_heads < 1 || c.kv_heads > 65536) return "pages and kv_heads must be at least 1, kv_heads at most 65536";
  if (c.page_size < 16 || c.page_size > 4096 || (c.page_size & (c.page_size - 1))) return "page_size must be a power of two, 16 to 4096";
  const bool e4m3 = c.dtype == TPS_E4M3;
  if (!c.k || !c.v) return "NULL cache";
  if (e4m3 != (c.exps != nullptr)) return "exps belong to TPS_E4M3, and to nothing else";
  if ((uintptr_t)c.k % 16 || (uintptr_t)c.v % 16 || (uintptr_t)c.exps % 4) return "the cache's values must start at 16-byte boundaries, exps at 4-byte ones";
  if (e4m3 && (int64_t)c.pages * 2 * c.kv_heads >= (1ll << 31) / c.page_size) return "pages 2 kv_heads page_size must be below 2^31";
  const int64_t n[3] = {c.pages, c.page_size, c.kv_heads}, bytes = e4m3 ? 1 : 2;
  for (int i = 0; i < 3; ++i) {
    const int64_t ks = n[i] > 1 ? c.k_stride[i] : 0, vs = n[i] > 1 ? c.v_stride[i] : 0;
    if (ks < 0 || vs < 0 || ks > kMostStride || vs > kMostStride || ks * bytes % 16 || vs * bytes % 16)
      return "the cache's strides must be whole 16 bytes, not negative, at most 2^40";
    if (n[i] > 1 && (ks < c.head_dim || vs < c.head_dim)) return "the cache's rows overlap";
    to->ks[i] = ks * bytes;
    to->vs[i] = vs * bytes;
  }
  if (to->ks[1] > bytes << 23 || to->vs[1] > bytes << 23 || (c.page_size - 1) * to->ks[1] >= bytes << 30 || (c.page_size - 1) * to->vs[1] >= bytes << 30)
    return "the cache's token strides must be at most 2^23, (page_size - 1) times them below 2^30";
  to->k = c.k;
  to->v = c.v;
  to->exps = c.exps;
  to->e4m3 = e4m3;
  to->pages = c.pages;
  to->heads = c.kv_heads;
  to->dim = c.head_dim;
  for (to->lg = 0; 1 << to->lg < c.page_size;) ++to->lg;
  return nullptr;
}

// The sequences. An error's text, or null.
const char* pages_of(const int32_t* table, int64_t stride, const int32_t* q_lens, const int32_t* kv_lens, int32_t batch, int32_t q_len,
                     int32_t max_pages, k::Pages* to) {
  if (!table || !kv_lens) return "NULL table or kv_lens";
  if ((uintptr_t)table % 4 || (uintptr_t)q_lens % 4 || (uintptr_t)kv_lens % 4) return "table or lengths not aligned to 4 bytes";
  if (max_pages < 1 || max_pages > kMostTokens) return "max_pages out of range";
  if (batch > 1 && (stride < 0 || stride > kMostStride)) return "table_stride out of range";
  *to = {table, batch > 1 ? stride : 0, q_lens, kv_lens, batch, q_len, max_pages};
  return nullptr;
}

// Strides of rows in elements: sequences, rows, heads. An error's text, or null.
const char* strides_of(const int64_t from[3], int64_t batch, int64_t rows, int64_t heads, int64_t least, int64_t to[3]) {
  const int64_t n[3] = {batch, rows, heads};
  for (int i = 0; i < 3; ++i) {
    const int64_t v = n[i] > 1 ? from[i] : 0;
    if (v < 0 || v % 8 || v > kMostStride) return "strides must be multiples of 8, not negative, below 2^40";
    if (n[i] > 1 && v < least) return "rows that are written overlap";
    to[i] = v;
  }
  return nullptr;
}

tp_status rows_call(const char* who, const tps_cache_rows_args* a, void* stream, bool append) {
  if (!a) return inval(who, "NULL arguments");
  k::CacheRows g;
  if (const char* e = cache_of(a->cache, &g.c)) return inval(who, e);
  if (a->reserved != 0) return inval(who, "reserved must be 0");
  if (a->batch < 0 || a->q_len < 0) return inval(who, "batch or q_len out of range");
  if (a->batch == 0 || a->q_len == 0) return ok();
  if (const char* e = pages_of(a->table, a->table_stride, a->q_lens, a->kv_lens, a->batch, a->q_len, a->max_pages, &g.p)) return inval(who, e);
  if (!a->k || !a->v) return inval(who, "NULL buffer");
  if ((uintptr_t)a->k % 16 || (uintptr_t)a->v % 16) return inval(who, "k and v must start at 16-byte boundaries");
  if ((int64_t)a->batch * a->q_len > ((1 << 26) - 1) / a->cache.kv_heads || (int64_t)a->batch * a->cache.kv_heads >= 1 << 22)
    return inval(who, "batch * q_len * kv_heads must be below 2^26, batch * kv_heads below 2^22");
  const int64_t least = append ? 0 : a->cache.head_dim;
  if (const char* e = strides_of(a->k_stride, a->batch, a->q_len, a->cache.kv_heads, least, g.rks)) return inval(who, e);
  if (const char* e = strides_of(a->v_stride, a->batch, a->q_len, a->cache.kv_heads, least, g.rvs)) return inval(who, e);
  g.k = static_cast<uint16_t*>(a->k);
  g.v = static_cast<uint16_t*>(a->v);
  hipStream_t s = static_cast<hipStream_t>(stream);
  OnDeviceOf dev(s);
  if (dev.error != hipSuccess) return done(who, dev.error);
  return done(who, append ? k::cache_append(g, s) : k::cache_read(g, s));
}

}  // namespace

extern "C" {

tp_status tps_cache_append(const tps_cache_rows_args* a, void* stream) { return rows_call("tps_cache_append", a, stream, true); }

tp_status tps_cache_read(const tps_cache_rows_args* a, void* stream) { return rows_call("tps_cache_read", a, stream, false); }

tp_status tps_cache_attention(const tps_cache_attention_args* a, void* stream) {
  static const char* who = "tps_cache_attention";
  if (!a) return inval(who, "NULL arguments");
  k::CacheAttention g;
  if (const char* e = cache_of(a->cache, &g.c)) return inval(who, e);
  if (a->batch < 0 || a->q_len < 0 || a->kv_len < 0 || a->kv_len > kMostTokens) return inval(who, "batch, q_len or kv_len out of range");
  if (a->heads < 1 || a->heads % a->cache.kv_heads || a->heads > 65536) return inval(who, "heads must be a multiple of kv_heads, at most 65536");
  if (a->sinks < 0) return inval(who, "sinks < 0");
  if (!(a->scale >= 0.f) || a->scale > 0x1p127f) return inval(who, "scale must be at most 2^127 and not negative");
  if ((uintptr_t)a->work % 256) return inval(who, "work must be 256-byte aligned");
  if (a->batch == 0 || a->q_len == 0) return ok();
  if (const char* e = pages_of(a->table, a->table_stride, a->q_lens, a->kv_lens, a->batch, a->q_len, a->max_pages, &g.p)) return inval(who, e);
  if (!a->q || !a->out) return inval(who, "NULL buffer");
  if ((uintptr_t)a->q % 16 || (uintptr_t)a->out % 16) return inval(who, "q and out must start at 16-byte boundaries");
  if ((int64_t)a->batch * a->q_len > ((1 << 27) - 1) / a->heads || (int64_t)a->batch * a->cache.kv_heads >= 1 << 22)
    return inval(who, "batch * q_len * heads must be below 2^27, batch * kv_heads below 2^22");
  if (const char* e = strides_of(a->q_stride, a->batch, a->q_len, a->heads, 0, g.qs)) return inval(who, e);
  if (const char* e = strides_of(a->out_stride, a->batch, a->q_len, a->heads, a->cache.head_dim, g.os)) return inval(who, e);
  g.q = static_cast<const uint16_t*>(a->q);
  g.out = static_cast<uint16_t*>(a->out);
  g.heads = a->heads;
  g.kv_len = (int)std::min<int64_t>(a->kv_len, (int64_t)a->max_pages * a->cache.page_size);
  g.window = a->window < 0 ? -1 : std::min(a->window, kMostTokens);
  g.sinks = a->sinks;
  g.scale = a->scale > 0.f ? a->scale : 1.f / std::sqrt((float)a->cache.head_dim);
  hipStream_t s = static_cast<hipStream_t>(stream);
  OnDeviceOf dev(s);
  if (dev.error != hipSuccess) return done(who, dev.error);
  return done(who, k::cache_attention(g, scratch(a->work, a->work_bytes), s));
}

tp_status tps_lora(const tps_lora_args* a, void* stream) {
  static const char* who = "tps_lora";
  if (!a) return inval(who, "NULL arguments");
  if (a->M < 0) return inval(who, "M < 0");
  if (a->N < 1 || a->K < 8 || a->K % 8 || a->K > 1 << 20) return inval(who, "need N >= 1 and K a multiple of 8 up to 2^20");
  if (a->R < 8 || a->R % 8 || a->R > 128) return inval(who, "R must be a multiple of 8 up to 128");
  if (a->adapters < 1) return inval(who, "adapters < 1");
  if (a->act < TP_ACT_NONE || a->act > TP_ACT_GELU) return inval(who, "unknown activation");
  if (a->dtype != TP_BF16 && a->dtype != TP_F32) return inval(who, "dtype must be TP_BF16 or TP_F32");
  if (a->reserved != 0) return inval(who, "reserved must be 0");
  if ((uintptr_t)a->work % 256) return inval(who, "work must be 256-byte aligned");
  if (a->M == 0) return ok();
  if (!a->x || !a->a || !a->b || !a->adapter || !a->y) return inval(who, "NULL buffer");
  if ((uintptr_t)a->x % 16 || (uintptr_t)a->a % 16 || (uintptr_t)a->b % 16) return inval(who, "x, a and b must start at 16-byte boundaries");
  if ((uintptr_t)a->adapter % 4 || (uintptr_t)a->ranks % 4 || (uintptr_t)a->scales % 4) return inval(who, "adapter, ranks or scales not aligned to 4 bytes");
  const uintptr_t item = a->dtype == TP_F32 ? 4 : 2;
  if ((uintptr_t)a->y % item || (uintptr_t)a->base % item) return inval(who, "y or base not aligned to its element");
  const bool many = a->M > 1, slots = a->adapters > 1;
  if (many && (a->ldx % 8 || a->ldx < a->K || a->ldx > kMostStride)) return inval(who, "ldx must be a multiple of 8, K or more, at most 2^40");
  if (many && (a->ldy < a->N || a->ldy > kMostStride)) return inval(who, "ldy must be N or more, at most 2^40");
  if (many && a->base && (a->ldbase < 0 || a->ldbase > kMostStride)) return inval(who, "ldbase must not be negative, at most 2^40");
  if (many && a->base == a->y && a->ldbase != a->ldy) return inval(who, "y may be base only with the same row stride");
  if (slots && (a->a_stride % 8 || a->b_stride % 8 || a->a_stride < 0 || a->b_stride < 0 || a->a_stride > kMostStride || a->b_stride > kMostStride))
    return inval(who, "a_stride and b_stride must be multiples of 8, not negative, at most 2^40");
  if (((int64_t)a->M + 15) / 16 * (((int64_t)a->N + 255) / 256) >= 1 << 24)
    return inval(who, "M in whole 16s times N in whole 256s must be below 2^36");
  k::Lora g;
  g.x = static_cast<const uint16_t*>(a->x);
  g.ldx = many ? a->ldx : 0;
  g.a = static_cast<const uint16_t*>(a->a);
  g.b = static_cast<const uint16_t*>(a->b);
  g.as = slots ? a->a_stride : 0;
  g.bs = slots ? a->b_stride : 0;
  g.adapter = a->adapter;
  g.ranks = a->ranks;
  g.scales = a->scales;
  g.base = a->base;
  g.ldbase = many ? a->ldbase : 0;
  g.y = a->y;
  g.ldy = many ? a->ldy : 0;
  g.f32 = a->dtype == TP_F32;
  g.M = a->M; g.N = a->N; g.K = a->K; g.R = a->R; g.adapters = a->adapters;
  g.act = a->act;
  hipStream_t s = static_cast<hipStream_t>(stream);
  OnDeviceOf dev(s);
  if (dev.error != hipSuccess) return done(who, dev.error);
  return done(who, k::lora(g, scratch(a->work, a->work_bytes), s));
}

}  // extern "C"
