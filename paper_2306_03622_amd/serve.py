"""ctypes binding of libtorpor's serving operators (include/torpor_serve.h): a paged key/value cache, attention over it, and
low-rank adapters of many requests. Argument marshalling only, in the manner of the operators in torpor.py."""
from __future__ import annotations

import ctypes as C
import struct

from .torpor import TP_ACT, TP_BF16, TP_F32, TP_OK, _P, _check, _stream_of, lib

TPS_E4M3 = 16


class tps_cache(C.Structure):
    _fields_ = [("k", C.c_void_p), ("v", C.c_void_p), ("exps", C.c_void_p), ("k_stride", C.c_int64 * 3), ("v_stride", C.c_int64 * 3),
                ("dtype", C.c_int32), ("pages", C.c_int32), ("page_size", C.c_int32), ("kv_heads", C.c_int32),
                ("head_dim", C.c_int32), ("reserved", C.c_int32)]


class tps_cache_rows_args(C.Structure):
    _fields_ = [("cache", tps_cache), ("table", C.c_void_p), ("table_stride", C.c_int64), ("q_lens", C.c_void_p),
                ("kv_lens", C.c_void_p), ("k", C.c_void_p), ("v", C.c_void_p), ("k_stride", C.c_int64 * 3), ("v_stride", C.c_int64 * 3),
                ("batch", C.c_int32), ("q_len", C.c_int32), ("max_pages", C.c_int32), ("reserved", C.c_int32)]


class tps_cache_attention_args(C.Structure):
    _fields_ = [("cache", tps_cache), ("table", C.c_void_p), ("table_stride", C.c_int64), ("q_lens", C.c_void_p),
                ("kv_lens", C.c_void_p), ("q", C.c_void_p), ("out", C.c_void_p), ("q_stride", C.c_int64 * 3), ("out_stride", C.c_int64 * 3),
                ("batch", C.c_int32), ("heads", C.c_int32), ("q_len", C.c_int32), ("kv_len", C.c_int32), ("max_pages", C.c_int32),
                ("window", C.c_int32), ("sinks", C.c_int32), ("scale", C.c_float), ("work", C.c_void_p), ("work_bytes", C.c_uint64)]


class tps_lora_args(C.Structure):
    _fields_ = [("x", C.c_void_p), ("ldx", C.c_int64), ("a", C.c_void_p), ("b", C.c_void_p), ("a_stride", C.c_int64),
                ("b_stride", C.c_int64), ("adapter", C.c_void_p), ("ranks", C.c_void_p), ("scales", C.c_void_p), ("base", C.c_void_p),
                ("ldbase", C.c_int64), ("y", C.c_void_p), ("ldy", C.c_int64), ("dtype", C.c_int32), ("M", C.c_int32), ("N", C.c_int32),
                ("K", C.c_int32), ("R", C.c_int32), ("adapters", C.c_int32), ("act", C.c_int32), ("reserved", C.c_int32),
                ("work", C.c_void_p), ("work_bytes", C.c_uint64)]


# Argument blocks are packed at once and handed over as bytes, a cache's part once for all its calls.
_CACHE = struct.Struct("@PPP6q6i")
_ROWS = struct.Struct("@PqPPPP6q4i")
_ATTENTION = struct.Struct("@PqPPPP6q7ifPQ")
_LORA = struct.Struct("@PqPPqqPPPPqPq8iPQ")
_calls = None


def _serve_calls():
    """(torch, its raw current stream by device, its current device, the library's calls on packed arguments)."""
    global _calls
    if _calls is None:
        import torch
        L, calls = lib(), []
        for name in ("tps_cache_append", "tps_cache_read", "tps_cache_attention", "tps_lora"):
            f = L[name]                   # a function object of its own
            f.argtypes, f.restype = [C.c_char_p, _P], C.c_int32
            calls.append(f)
        _calls = (torch, torch._C._cuda_getCurrentRawStream, torch._C._cuda_getDevice, *calls)
    return _calls


def _made(torch, current, here, call, packed, dev, stream):
    """Makes the call on `stream` (None: the device's current one) with the tensors' device the current one where that matters."""
    s = current(dev) if stream is None else _stream_of(dev, stream)
    if s or here() == dev:                # the null stream is that of whichever device is current; any other carries its own
        status = call(packed, s)
    else:
        with torch.cuda.device(dev):
            status = call(packed, s)
    if status != TP_OK:
        _check(lib(), status)


def _ints(name, t, n, torch, dev):
    """Address of a contiguous int32 [n] on the device."""
    if t.dtype is not torch.int32 or t.shape != (n,) or not t.is_contiguous() or t.get_device() != dev:
        raise ValueError(f"{name} must be a contiguous int32 [{n}] on device {dev}, not {t.dtype} {tuple(t.shape)} on {t.device}")
    return t.data_ptr()


def _scratch(t, dev):
    """Address and bytes of a scratch tensor."""
    if t.get_device() != dev or not t.is_contiguous():
        raise ValueError(f"work must be contiguous and on device {dev}, not {tuple(t.shape)} by {t.stride()} on {t.device}")
    return t.data_ptr(), t.numel() * t.element_size()


class PagedCache:
    """A pool of pages of keys and values on the device: k, v [pages][page_size][kv_heads][dim], bf16, or 8-bit (float8_e4m3fn or
    uint8) with exps uint8 [pages][2][kv_heads][page_size]; any strides but the last. It shares the memory of the tensors
    it is made from and keeps that memory; a call goes by the addresses taken here."""

    __slots__ = ("_k", "_v", "_exps", "_packed", "device", "pages", "page_size", "kv_heads", "head_dim", "e4m3")

    def __init__(self, k, v, exps=None):
        import torch
        if k.dim() != 4 or v.shape != k.shape or v.dtype != k.dtype:
            raise ValueError(f"k {k.dtype} {tuple(k.shape)}, v {v.dtype} {tuple(v.shape)}")
        e4m3 = k.dtype in (torch.float8_e4m3fn, torch.uint8)
        if not e4m3 and k.dtype != torch.bfloat16:
            raise ValueError(f"k and v must be bfloat16, float8_e4m3fn or uint8, not {k.dtype}")
        pages, size, heads, dim = k.shape
        if k.device.type != "cuda" or v.device != k.device:
            raise ValueError(f"k on {k.device}, v on {v.device}")
        if k.stride(3) != 1 or v.stride(3) != 1:
            raise ValueError("the values of a head must be contiguous")
        if e4m3 != (exps is not None):
            raise ValueError("exps belong to 8-bit keys and values, and to nothing else")
        if e4m3 and (exps.dtype != torch.uint8 or tuple(exps.shape) != (pages, 2, heads, size) or not exps.is_contiguous() or
                     exps.device != k.device):
            raise ValueError(f"exps must be a contiguous uint8 {(pages, 2, heads, size)} on {k.device}, not {exps.dtype} {tuple(exps.shape)} on {exps.device}")
        packed = _CACHE.pack(k.data_ptr(), v.data_ptr(), exps.data_ptr() if e4m3 else 0, *k.stride()[:3], *v.stride()[:3],
                             TPS_E4M3 if e4m3 else TP_BF16, pages, size, heads, dim, 0)
        # tensor objects of its own hold the memory: the caller's may be given other memory (t.data = ..)
        for name, value in (("_k", k.detach()), ("_v", v.detach()), ("_exps", exps.detach() if e4m3 else None), ("device", k.device),
                            ("_packed", (k.device.index, packed)), ("pages", pages), ("page_size", size), ("kv_heads", heads),
                            ("head_dim", dim), ("e4m3", e4m3)):
            object.__setattr__(self, name, value)

    def __setattr__(self, name, value):
        raise AttributeError(f"{name} of a PagedCache is fixed: make another one")

    def __reduce__(self):                 # copies and pickles: made anew from its tensors
        return PagedCache, (self._k, self._v, self._exps)

    k = property(lambda self: self._k.detach())
    v = property(lambda self: self._v.detach())
    exps = property(lambda self: None if self._exps is None else self._exps.detach())

    @classmethod
    def empty(cls, pages: int, page_size: int, kv_heads: int, head_dim: int, e4m3: bool = False, device="cuda"):
        """A pool whose places hold nothing yet."""
        import torch
        k, v = (torch.empty(pages, page_size, kv_heads, head_dim, dtype=torch.float8_e4m3fn if e4m3 else torch.bfloat16, device=device) for _ in "kv")
        return cls(k, v, torch.empty(pages, 2, kv_heads, page_size, dtype=torch.uint8, device=device) if e4m3 else None)


def _table(table, batch, torch, dev):
    """(address, row stride, columns) of a table of pages."""
    if table.dtype is not torch.int32 or table.dim() != 2 or table.shape[0] != batch or table.get_device() != dev:
        raise ValueError(f"table must be int32 [{batch}][pages] on device {dev}, not {table.dtype} {tuple(table.shape)} on {table.device}")
    if table.shape[1] > 1 and table.stride(1) != 1:
        raise ValueError("table: rows must be contiguous")
    return table.data_ptr(), table.stride(0), table.shape[1]


def _heads(name, t, bf, dev):
    """Raises for a tensor of heads that a call cannot take."""
    if t.dtype is not bf:
        raise ValueError(f"{name} is {t.dtype}")
    if t.get_device() != dev:
        raise ValueError(f"{name} is on {t.device}, the cache on device {dev}")
    if t.stride(3) != 1:
        raise ValueError(f"{name}: the values of a head must be contiguous")


def _rows(which, cache, table, kv_lens, k, v, q_lens, stream):
    calls = _calls or _serve_calls()
    torch, current, here = calls[:3]
    dev, packed = cache._packed
    if k.dim() != 4 or v.shape != k.shape or k.shape[2] != cache.kv_heads or k.shape[3] != cache.head_dim:
        raise ValueError(f"k {tuple(k.shape)}, v {tuple(v.shape)}, a cache of {cache.kv_heads} heads of {cache.head_dim}")
    b, n = k.shape[:2]
    for name, t in (("k", k), ("v", v)):
        _heads(name, t, torch.bfloat16, dev)
    tp, ts, columns = _table(table, b, torch, dev)
    kl = _ints("kv_lens", kv_lens, b, torch, dev)
    ql = 0 if q_lens is None else _ints("q_lens", q_lens, b, torch, dev)
    k0, k1, k2, _ = k.stride()
    v0, v1, v2, _ = v.stride()
    packed += _ROWS.pack(tp, ts, ql, kl, k.data_ptr(), v.data_ptr(), k0, k1, k2, v0, v1, v2, b, n, columns, 0)
    _made(torch, current, here, calls[which], packed, dev, stream)


def tps_cache_append(cache: PagedCache, table, kv_lens, k, v, q_lens=None, stream=None):
    """Writes the new tokens' k, v [B][q_len][kv_heads][dim] (bf16, any strides but the last) into the pages: the last q_lens[b]
    (default q_len) of sequence b's kv_lens[b] tokens. table int32 [B][pages a sequence], lengths int32 [B], on the device."""
    _rows(3, cache, table, kv_lens, k, v, q_lens, stream)


def tps_cache_read(cache: PagedCache, table, kv_lens, k, v, q_lens=None, stream=None):
    """Reads the last q_lens[b] (default q_len) tokens of each sequence into k, v [B][q_len][kv_heads][dim], bf16; the reverse of
    tps_cache_append."""
    _rows(4, cache, table, kv_lens, k, v, q_lens, stream)


def tps_cache_attention(cache: PagedCache, table, kv_lens, q, out, q_lens=None, kv_len: int | None = None, window: int = -1, sinks: int = 0,
                        scale: float = 0.0, work=None, stream=None):
    """Attention of the new tokens' q [B][q_len][heads][dim] over the cache, which holds their keys and values already, into out
    (as q), bf16, in causal order. kv_len: no sequence is longer (default: what the table has room for); window: keys to the
    left of a token that it sees (negative: all); sinks: first keys that it sees besides; see torpor_serve.h."""
    calls = _calls or _serve_calls()
    torch, current, here = calls[:3]
    dev, packed = cache._packed
    if q.dim() != 4 or out.shape != q.shape or q.shape[3] != cache.head_dim:
        raise ValueError(f"q {tuple(q.shape)}, out {tuple(out.shape)}, a cache of heads of {cache.head_dim}")
    b, n, h, _ = q.shape
    q0, q1, q2, q3 = q.stride()
    o0, o1, o2, o3 = out.stride()
    bf = torch.bfloat16
    if not (q.dtype is out.dtype is bf and q3 == o3 == 1 and q.get_device() == out.get_device() == dev):
        for name, t in (("q", q), ("out", out)):
            _heads(name, t, bf, dev)
    tp, ts, columns = _table(table, b, torch, dev)
    kl = _ints("kv_lens", kv_lens, b, torch, dev)
    ql = 0 if q_lens is None else _ints("q_lens", q_lens, b, torch, dev)
    wp, wb = (0, 0) if work is None else _scratch(work, dev)
    packed += _ATTENTION.pack(tp, ts, ql, kl, q.data_ptr(), out.data_ptr(), q0, q1, q2, o0, o1, o2, b, h, n,
                              columns * cache.page_size if kv_len is None else kv_len, columns, window, sinks, scale, wp, wb)
    _made(torch, current, here, calls[5], packed, dev, stream)


def tps_lora(x, a, b, adapter, out, base=None, ranks=None, scales=None, act: str = "none", work=None, stream=None):
    """out[m] = act(base[m] + scales[i] b[i] (a[i] x[m])), i = adapter[m] (outside the pool: none): x bf16 [M][K], a bf16
    [adapters][R][K], b bf16 [adapters][N][R], adapter int32 [M], out and base bf16 or fp32 [M][N] (base may be out; default zeros),
    ranks int32 [adapters] (default R), scales fp32 [adapters] (default 1), all on x's device."""
    torch, current, here, _, _, _, call = _calls or _serve_calls()
    bf, dev = torch.bfloat16, x.get_device()
    if dev < 0:
        raise ValueError(f"x on {x.device}")
    if x.dim() != 2 or a.dim() != 3 or b.dim() != 3 or out.dim() != 2:
        raise ValueError(f"x {tuple(x.shape)}, a {tuple(a.shape)}, b {tuple(b.shape)}, out {tuple(out.shape)}")
    m, k = x.shape
    slots, r, ka = a.shape
    n = out.shape[1]
    if ka != k or b.shape != (slots, n, r) or out.shape[0] != m:
        raise ValueError(f"x {tuple(x.shape)}, a {tuple(a.shape)}, b {tuple(b.shape)}, out {tuple(out.shape)}")
    f32 = out.dtype is torch.float32
    a0, a1, a2 = a.stride()
    b0, b1, b2 = b.stride()
    if not (x.dtype is a.dtype is b.dtype is bf and (f32 or out.dtype is bf)):
        raise ValueError(f"x {x.dtype}, a {a.dtype}, b {b.dtype}, out {out.dtype}")
    if not (a.get_device() == b.get_device() == out.get_device() == dev):
        raise ValueError(f"x on device {dev}, a on {a.device}, b on {b.device}, out on {out.device}")
    if (k > 1 and x.stride(1) != 1) or (n > 1 and out.stride(1) != 1):
        raise ValueError("rows of x and out must be contiguous")
    if a2 != 1 or b2 != 1 or a1 != k or (n > 1 and b1 != r):
        raise ValueError("every adapter's matrices must be contiguous")
    bp = ldb = rp = sp = wp = wb = 0
    if base is not None:
        if base.dtype is not out.dtype or base.shape != out.shape or base.get_device() != dev or (n > 1 and base.stride(1) != 1):
            raise ValueError(f"base must be {out.dtype} {tuple(out.shape)} with contiguous rows on device {dev}")
        bp, ldb = base.data_ptr(), base.stride(0)
    ap = _ints("adapter", adapter, m, torch, dev)
    if ranks is not None:
        rp = _ints("ranks", ranks, slots, torch, dev)
    if scales is not None:
        if scales.dtype is not torch.float32 or scales.shape != (slots,) or not scales.is_contiguous() or scales.get_device() != dev:
            raise ValueError(f"scales must be a contiguous float32 [{slots}] on device {dev}")
        sp = scales.data_ptr()
    if work is not None:
        wp, wb = _scratch(work, dev)
    packed = _LORA.pack(x.data_ptr(), x.stride(0), a.data_ptr(), b.data_ptr(), a0, b0, ap, rp, sp, bp, ldb, out.data_ptr(), out.stride(0),
                        TP_F32 if f32 else TP_BF16, m, n, k, r, slots, TP_ACT[act], 0, wp, wb)
    _made(torch, current, here, call, packed, dev, stream)
