// The operators' C entry points (torpor_ops.h): argument checks, the device of the stream, the launch.
#include <cmath>

#include "../core/w4.hpp"
#include "ops_common.hpp"
#include "torpor_ops.h"

using namespace tp;

extern "C" {

tp_status tpo_linear_w4(const tpo_linear_w4_args* a, void* stream) {
  static const char* who = "tpo_linear_w4";
  if (!a) return inval(who, "NULL arguments");
  if (a->M < 0) return inval(who, "M < 0");
  if (!w4_shape_ok(a->N, a->K, a->group))
    return inval(who, "need 1 <= N <= 2^24, 1 <= K <= 2^20, group 32, 64 or 128 dividing K");
  if (a->act < TP_ACT_NONE || a->act > TP_ACT_GELU) return inval(who, "unknown activation");
  if (a->y_dtype != TP_BF16 && a->y_dtype != TP_F32) return inval(who, "y_dtype must be TP_BF16 or TP_F32");
  if ((uintptr_t)a->work % 256) return inval(who, "work must be 256-byte aligned");
  if (a->M == 0) return ok();
  if (!a->x || !a->wq || !a->scales || !a->y) return inval(who, "NULL buffer");
  if ((uintptr_t)a->x % 16 || a->ldx % 8) return inval(who, "x must start at a 16-byte boundary, ldx be a multiple of 8");
  if ((uintptr_t)a->wq % 16 || (uintptr_t)a->scales % 16) return inval(who, "wq and scales must start at 16-byte boundaries");
  if ((uintptr_t)a->y % (a->y_dtype == TP_F32 ? 4 : 2) || (uintptr_t)a->bias % 2 || (uintptr_t)a->res % 2)
    return inval(who, "y, bias or res not aligned to its element");
  if (a->ldx < a->K || a->ldy < a->N || (a->res && a->ldr < a->N)) return inval(who, "a row stride below the row's length");
  if (a->ldx >= 1 << 23 || a->ldy > kMostStride || (a->res && a->ldr > kMostStride)) return inval(who, "row stride too large");
  if (((int64_t)a->M + 127) / 128 * ((a->N + 255) / 256) >= 1 << 23)
    return inval(who, "M in whole 128s times N in whole 256s must be below 2^38");
  if (a->res == a->y && (a->y_dtype != TP_BF16 || a->ldr != a->ldy))
    return inval(who, "y may be res only in bf16 and with the same row stride");
  k::LinearW4 g;
  g.x = static_cast<const uint16_t*>(a->x);
  g.ldx = a->ldx;
  g.wq = static_cast<const uint8_t*>(a->wq);
  g.scales = static_cast<const uint16_t*>(a->scales);
  g.bias = static_cast<const uint16_t*>(a->bias);
  g.res = static_cast<const uint16_t*>(a->res);
  g.ldr = a->ldr;
  g.y = a->y;
  g.ldy = a->ldy;
  g.y_f32 = a->y_dtype == TP_F32;
  g.M = a->M; g.N = a->N; g.K = a->K; g.group = a->group; g.act = a->act;
  hipStream_t s = static_cast<hipStream_t>(stream);
  OnDeviceOf dev(s);
  if (dev.error != hipSuccess) return done(who, dev.error);
  return done(who, k::linear_w4(g, s));
}

tp_status tpo_attention(const tpo_attention_args* a, void* stream) {
  static const char* who = "tpo_attention";
  if (!a) return inval(who, "NULL arguments");
  if (a->batch < 0 || a->q_len < 0 || a->kv_len < 0 || a->batch > kMostTokens || a->q_len > kMostTokens || a->kv_len > kMostTokens)
    return inval(who, "batch, q_len or kv_len out of range");
  if (a->heads < 1 || a->kv_heads < 1 || a->heads % a->kv_heads || a->heads > 65536)
    return inval(who, "heads must be a multiple of kv_heads, both at least 1");
  if (a->head_dim != 64 && a->head_dim != 128) return inval(who, "head_dim must be 64 or 128");
  if (a->causal != 0 && a->causal != 1) return inval(who, "causal must be 0 or 1");
  if (a->sinks < 0) return inval(who, "sinks < 0");
  // (the kernels multiply by scale log2(e), which has to be finite too)
  if (!(a->scale >= 0.f) || a->scale > 0x1p127f) return inval(who, "scale must be at most 2^127 and not negative");
  if ((uintptr_t)a->work % 256) return inval(who, "work must be 256-byte aligned");
  if (a->batch == 0 || a->q_len == 0) return ok();
  if (!a->q || !a->out || (a->kv_len > 0 && (!a->k || !a->v))) return inval(who, "NULL buffer");
  for (const void* p : {a->q, a->k, a->v, static_cast<const void*>(a->out)})
    if ((uintptr_t)p % 16) return inval(who, "q, k, v and out must start at 16-byte boundaries");
  if ((uintptr_t)a->q_lens % 4 || (uintptr_t)a->kv_lens % 4) return inval(who, "lengths not aligned to 4 bytes");
  // strides of dimensions of one entry are not used
  const int64_t nq[3] = {a->batch, a->q_len, a->heads}, nk[3] = {a->batch, a->kv_len, a->kv_heads};
  k::Attention g;
  const struct {
    const int64_t *from, *n;
    int64_t* to;
  } strides[4] = {{a->q_stride, nq, g.qs}, {a->k_stride, nk, g.ks}, {a->v_stride, nk, g.vs}, {a->out_stride, nq, g.os}};
  for (const auto& st : strides)
    for (int i = 0; i < 3; ++i) {
      const int64_t v = st.n[i] > 1 ? st.from[i] : 0;
      if (v < 0 || v % 8 || v > kMostStride) return inval(who, "strides must be multiples of 8, not negative, below 2^40");
      if (st.to == g.os && st.n[i] > 1 && v < a->head_dim) return inval(who, "out rows overlap");
      st.to[i] = v;
    }
  if (g.ks[1] > 1 << 23 || g.vs[1] > 1 << 23) return inval(who, "token strides of k and v must be at most 2^23");
  if ((int64_t)a->q_len * a->heads * a->batch >= 1ll << 30 || (int64_t)a->batch * a->kv_heads >= 1 << 22)
    return inval(who, "batch * q_len * heads must be below 2^30, batch * kv_heads below 2^22");
  g.q = static_cast<const uint16_t*>(a->q);
  g.k = static_cast<const uint16_t*>(a->k);
  g.v = static_cast<const uint16_t*>(a->v);
  g.out = static_cast<uint16_t*>(a->out);
  g.q_lens = a->q_lens;
  g.kv_lens = a->kv_lens;
  g.batch = a->batch; g.heads = a->heads; g.kv_heads = a->kv_heads; g.dim = a->head_dim;
  g.q_len = a->q_len; g.kv_len = a->kv_len;
  g.causal = a->causal;
  g.left = a->window_left < 0 ? -1 : a->window_left > kMostTokens ? kMostTokens : a->window_left;
  g.right = a->window_right < 0 ? -1 : a->window_right > kMostTokens ? kMostTokens : a->window_right;
  g.sinks = a->sinks;
  g.scale = a->scale > 0.f ? a->scale : 1.f / std::sqrt((float)a->head_dim);
  hipStream_t s = static_cast<hipStream_t>(stream);
  OnDeviceOf dev(s);
  if (dev.error != hipSuccess) return done(who, dev.error);
  return done(who, k::attention_masked(g, scratch(a->work, a->work_bytes), s));
}

}  // extern "C"
