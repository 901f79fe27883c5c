"""ctypes binding of libtorpor's serving operators (include/torpor_serve.h): a paged key/value cache, attention over it, and
low-rank adapters of many requests. Argument marshalling only, in the manner of the operators in torpor.py."""
from __future__ import annotations

import ctypes as C
import struct

from .torpor import TP_ACT, TP_BF16, TP_F32, TP_OK, _P, _check, _stream_of, lib

TPS_E4M3 = 16
_MOST_TOKENS = (1 << 30) - 1              # of a sequence


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


def _on_device(torch, call, packed, dev, stream):
    """The call's status, made with the tensors' device the current one."""
    with torch.cuda.device(dev):
        return call(packed, stream)


# What the calls check they check in place, all at once, since a function call for each tensor took 1 us of a 6.5 us call; the functions
# below then say what is wrong.

def _ints(name, t, n, torch, dev):
    if t.dtype is not torch.int32 or t.numel() != n or not t.is_contiguous() or t.get_device() != dev:
        raise ValueError(f"{name} must be a contiguous int32 [{n}] on device {dev}, not {t.dtype} {tuple(t.shape)} on {t.device}")


def _scratch(t, dev):
    """Address and bytes of a scratch tensor."""
    if t.get_device() != dev or not t.is_contiguous():
        raise ValueError(f"work must be contiguous and on device {dev}, not {tuple(t.shape)} by {t.stride()} on {t.device}")
    return t.data_ptr(), t.numel() * t.element_size()


def _heads(name, t, bf, dev):
    if t.dtype is not bf:
        raise ValueError(f"{name} is {t.dtype}")
    if t.get_device() != dev:
        raise ValueError(f"{name} is on {t.device}, the cache on device {dev}")
    if t.stride(3) != 1:
        raise ValueError(f"{name}: the values of a head must be contiguous")


def _wrong(torch, dev, batch, table, kv_lens, q_lens, **heads):
    """Raises for the first of the tensors that a call on a cache cannot take."""
    for name, t in heads.items():
        _heads(name, t, torch.bfloat16, dev)
    if table.dtype is not torch.int32 or table.dim() != 2 or table.shape[0] != batch or table.get_device() != dev:
        raise ValueError(f"table must be int32 [{batch}][pages] on device {dev}, not {table.dtype} {tuple(table.shape)} on {table.device}")
    if table.shape[1] > 1 and table.stride(1) != 1:
        raise ValueError("table: rows must be contiguous")
    _ints("kv_lens", kv_lens, batch, torch, dev)
    if q_lens is not None:
        _ints("q_lens", q_lens, batch, torch, dev)


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
                            ("_packed", (k.device.index, packed, heads, dim, size)), ("pages", pages), ("page_size", size), ("kv_heads", heads),
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


def _rows(which, cache, table, kv_lens, k, v, q_lens, stream):
    calls = _calls or _serve_calls()
    torch, current, here = calls[:3]
    dev, packed, heads, dim, _ = cache._packed
    shape = k.shape
    if len(shape) != 4 or v.shape != shape or shape[2] != heads or shape[3] != dim:
        raise ValueError(f"k {tuple(k.shape)}, v {tuple(v.shape)}, a cache of {heads} heads of {dim}")
    b, n = shape[0], shape[1]
    bf, i32 = torch.bfloat16, torch.int32
    k0, k1, k2, k3 = k.stride()
    v0, v1, v2, v3 = v.stride()
    if not (k.dtype is v.dtype is bf and table.dtype is kv_lens.dtype is i32 and k3 == v3 == 1 and table.dim() == 2 and
            k.get_device() == v.get_device() == table.get_device() == kv_lens.get_device() == dev and kv_lens.numel() == b and
            kv_lens.is_contiguous() and table.shape[0] == b and table.stride(1) == 1 and
            (q_lens is None or (q_lens.dtype is i32 and q_lens.numel() == b and q_lens.is_contiguous() and q_lens.get_device() == dev))):
        _wrong(torch, dev, b, table, kv_lens, q_lens, k=k, v=v)
    columns = table.shape[1]
    packed += _ROWS.pack(table.data_ptr(), table.stride(0), 0 if q_lens is None else q_lens.data_ptr(), kv_lens.data_ptr(), k.data_ptr(),
                         v.data_ptr(), k0, k1, k2, v0, v1, v2, b, n, columns, 0)
    s = current(dev) if stream is None else _stream_of(dev, stream)
    # the null stream is that of whichever device is current; any other carries its own
    status = calls[which](packed, s) if s or here() == dev else _on_device(torch, calls[which], packed, dev, s)
    if status != TP_OK:
        _check(lib(), status)


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
    (as q), bf16, in causal order. kv_len: no sequence is longer (default: what the table has room for, up to 2^30 - 1); window: keys to the
    left of a token that it sees (negative: all); sinks: first keys that it sees besides; see torpor_serve.h."""
    torch, current, here, _, _, call, _ = _calls or _serve_calls()
    dev, packed, _, dim, size = cache._packed
    shape = q.shape
    if len(shape) != 4 or out.shape != shape or shape[3] != dim:
        raise ValueError(f"q {tuple(q.shape)}, out {tuple(out.shape)}, a cache of heads of {dim}")
    b, n, h, _ = shape
    q0, q1, q2, q3 = q.stride()
    o0, o1, o2, o3 = out.stride()
    i32 = torch.int32
    if not (q.dtype is out.dtype is torch.bfloat16 and table.dtype is kv_lens.dtype is i32 and q3 == o3 == 1 and table.dim() == 2 and
            q.get_device() == out.get_device() == table.get_device() == kv_lens.get_device() == dev and kv_lens.numel() == b and
            kv_lens.is_contiguous() and table.shape[0] == b and table.stride(1) == 1 and
            (q_lens is None or (q_lens.dtype is i32 and q_lens.numel() == b and q_lens.is_contiguous() and q_lens.get_device() == dev))):
        _wrong(torch, dev, b, table, kv_lens, q_lens, q=q, out=out)
    columns = table.shape[1]
    wp, wb = (0, 0) if work is None else _scratch(work, dev)
    packed += _ATTENTION.pack(table.data_ptr(), table.stride(0), 0 if q_lens is None else q_lens.data_ptr(), kv_lens.data_ptr(), q.data_ptr(),
                              out.data_ptr(), q0, q1, q2, o0, o1, o2, b, h, n, min(columns * size, _MOST_TOKENS) if kv_len is None else kv_len, columns, window,
                              sinks, scale, wp, wb)
    s = current(dev) if stream is None else _stream_of(dev, stream)
    status = call(packed, s) if s or here() == dev else _on_device(torch, call, packed, dev, s)
    if status != TP_OK:
        _check(lib(), status)


def tps_lora(x, a, b, adapter, out, base=None, ranks=None, scales=None, act: str = "none", work=None, stream=None):
    """out[m] = act(base[m] + scales[i] b[i] (a[i] x[m])), i = adapter[m] (outside the pool: none): x bf16 [M][K], a bf16
    [adapters][R][K], b bf16 [adapters][N][R], adapter int32 [M], out and base bf16 or fp32 [M][N] (base may be out; default zeros),
    ranks int32 [adapters] (default R), scales fp32 [adapters] (default 1), all on x's device."""
    torch, current, here, _, _, _, call = _calls or _serve_calls()
    bf, dev = torch.bfloat16, x.get_device()
    if dev < 0:
        raise ValueError(f"x on {x.device}")
    xs, ash, os = x.shape, a.shape, out.shape
    if len(xs) != 2 or len(ash) != 3 or len(os) != 2 or ash[2] != xs[1] or os[0] != xs[0] or b.shape != (ash[0], os[1], ash[1]):
        raise ValueError(f"x {tuple(x.shape)}, a {tuple(a.shape)}, b {tuple(b.shape)}, out {tuple(out.shape)}")
    m, k = xs
    slots, r, _ = ash
    n = os[1]
    f32 = out.dtype is torch.float32
    a0, a1, a2 = a.stride()
    b0, b1, b2 = b.stride()
    x0, x1 = x.stride()
    o0, o1 = out.stride()
    if not (x.dtype is a.dtype is b.dtype is bf and (f32 or out.dtype is bf)):
        raise ValueError(f"x {x.dtype}, a {a.dtype}, b {b.dtype}, out {out.dtype}")
    if not (a.get_device() == b.get_device() == out.get_device() == dev):
        raise ValueError(f"x on device {dev}, a on {a.device}, b on {b.device}, out on {out.device}")
    if x1 != 1 or (o1 != 1 and n > 1):
        raise ValueError("rows of x and out must be contiguous")
    if a2 != 1 or b2 != 1 or a1 != k or (b1 != r and n > 1):
        raise ValueError("every adapter's matrices must be contiguous")
    bp = ldb = rp = sp = wp = wb = 0
    if base is not None:
        ldb, base1 = base.stride() if base.dim() == 2 else (0, 0)
        if base.dtype is not out.dtype or base.shape != os or base.get_device() != dev or (base1 != 1 and n > 1):
            raise ValueError(f"base must be {out.dtype} {tuple(out.shape)} with contiguous rows on device {dev}")
        bp = base.data_ptr()
    if adapter.dtype is not torch.int32 or adapter.numel() != m or not adapter.is_contiguous() or adapter.get_device() != dev:
        _ints("adapter", adapter, m, torch, dev)
    if ranks is not None:
        _ints("ranks", ranks, slots, torch, dev)
        rp = ranks.data_ptr()
    if scales is not None:
        if scales.dtype is not torch.float32 or scales.numel() != slots or not scales.is_contiguous() or scales.get_device() != dev:
            raise ValueError(f"scales must be a contiguous float32 [{slots}] on device {dev}")
        sp = scales.data_ptr()
    if work is not None:
        wp, wb = _scratch(work, dev)
    packed = _LORA.pack(x.data_ptr(), x0, a.data_ptr(), b.data_ptr(), a0, b0, adapter.data_ptr(), rp, sp, bp, ldb, out.data_ptr(), o0,
                        TP_F32 if f32 else TP_BF16, m, n, k, r, slots, TP_ACT[act], 0, wp, wb)
    s = current(dev) if stream is None else _stream_of(dev, stream)
    status = call(packed, s) if s or here() == dev else _on_device(torch, call, packed, dev, s)
    if status != TP_OK:
        _check(lib(), status)
