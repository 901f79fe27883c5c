"""The serving operators' host side (no GPU): exported symbols, struct layouts, every refusal of invalid arguments, which comes
before any launch, and what the binding hands to the library."""
import contextlib
import copy
import ctypes
import os
import re
import shutil
import subprocess
import types

import numpy as np
import pytest

import paper_2306_03622_amd as tp
from paper_2306_03622_amd import serve as S
from paper_2306_03622_amd import torpor as T
from tests.serve_common import e4m3_rows, e4m3_values

torch = pytest.importorskip("torch")
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
NAMES = {"tps_cache_append", "tps_cache_read", "tps_cache_attention", "tps_lora"}


def test_library_exports_the_serving_header():
    src = open(os.path.join(ROOT, "include", "torpor_serve.h")).read()
    declared = set(re.findall(r"^TP_API\s+[\w\s\*]+?\b(tps_\w+)\s*\(", src, re.M))
    assert declared == NAMES
    out = subprocess.run(["nm", "-D", "--defined-only", T.LIB_PATH], capture_output=True, text=True).stdout
    assert set(re.findall(r" T (tps_\w+)", out)) == declared
    assert int(re.search(r"#define TPS_E4M3 (\d+)", src).group(1)) == tp.TPS_E4M3


@pytest.mark.parametrize("name", ["tps_cache", "tps_cache_rows_args", "tps_cache_attention_args", "tps_lora_args"])
def test_ctypes_layout_matches_the_header(name, tmp_path):
    cc = shutil.which("gcc") or shutil.which("cc")
    if not cc:
        pytest.skip("no C compiler")
    cls = getattr(S, name)
    src = ["#include <stdio.h>", "#include <stddef.h>", '#include "torpor_serve.h"', "int main(void) {",
           f'  printf("size %zu\\n", sizeof({name}));']
    src += [f'  printf("{f} %zu\\n", offsetof({name}, {f}));' for f, _ in cls._fields_] + ["  return 0;", "}"]
    (tmp_path / "l.c").write_text("\n".join(src) + "\n")
    subprocess.run([cc, "-std=c11", "-I", os.path.join(ROOT, "include"), str(tmp_path / "l.c"), "-o", str(tmp_path / "l")], check=True)
    got = dict(l.split() for l in subprocess.run([str(tmp_path / "l")], check=True, capture_output=True, text=True).stdout.splitlines())
    assert int(got.pop("size")) == ctypes.sizeof(cls)
    assert {f: int(v) for f, v in got.items()} == {f: getattr(cls, f).offset for f, _ in cls._fields_}


def _flat(a):
    out = []
    for name, _ in a._fields_:
        v = getattr(a, name)
        out += _flat(v) if isinstance(v, ctypes.Structure) else list(v) if hasattr(v, "__len__") else [v]
    return out


def test_packed_arguments_have_the_structs_layout():
    head = list(range(1, 16))
    assert _flat(S.tps_cache.from_buffer_copy(S._CACHE.pack(*head))) == head
    for packer, cls, values in ((S._ROWS, S.tps_cache_rows_args, list(range(20, 36))),
                                (S._ATTENTION, S.tps_cache_attention_args, [*range(20, 39), 0.5, 40, 41])):
        assert S._CACHE.size + packer.size == ctypes.sizeof(cls)
        assert _flat(cls.from_buffer_copy(S._CACHE.pack(*head) + packer.pack(*values))) == head + values
    assert S._LORA.size == ctypes.sizeof(S.tps_lora_args)
    assert _flat(S.tps_lora_args.from_buffer_copy(S._LORA.pack(*range(1, 24)))) == list(range(1, 24))


def _status(name, args):
    L = tp.lib()
    f = L[name]
    f.argtypes, f.restype = [ctypes.c_void_p, ctypes.c_void_p], ctypes.c_int32
    st = f(None if args is None else ctypes.addressof(args), None)
    return st, L.tp_last_error().decode()


def _set(a, kw):
    for k, v in kw.items():
        obj, name = (a.cache, k[2:]) if k.startswith("c_") else (a, k)
        if isinstance(v, (tuple, list)):
            v = (ctypes.c_int64 * 3)(*v)
        setattr(obj, name, v)
    return a


# (addresses below are never read: every call here is refused before a launch)
def _cache(e4m3=False):
    return S.tps_cache(k=0x10000, v=0x20000, exps=0x30000 if e4m3 else None, k_stride=(16 * 2 * 64, 2 * 64, 64), v_stride=(16 * 2 * 64, 2 * 64, 64),
                       dtype=tp.TPS_E4M3 if e4m3 else tp.TP_BF16, pages=8, page_size=16, kv_heads=2, head_dim=64)


def rows_args(e4m3=False, **kw):
    return _set(S.tps_cache_rows_args(cache=_cache(e4m3), table=0x1000, table_stride=4, q_lens=None, kv_lens=0x2000, k=0x4000, v=0x5000,
                                      k_stride=(128 * 3, 128, 64), v_stride=(128 * 3, 128, 64), batch=2, q_len=3, max_pages=4), kw)


def attention_args(e4m3=False, **kw):
    return _set(S.tps_cache_attention_args(cache=_cache(e4m3), table=0x1000, table_stride=4, q_lens=None, kv_lens=0x2000, q=0x4000, out=0x5000,
                                           q_stride=(256 * 3, 256, 64), out_stride=(256 * 3, 256, 64), batch=2, heads=4, q_len=3, kv_len=64,
                                           max_pages=4, window=-1), kw)


BAD_CACHE = [
    {"c_dtype": 0}, {"c_dtype": 2}, {"c_dtype": tp.TPS_E4M3}, {"c_exps": 0x30000}, {"c_reserved": 1}, {"c_head_dim": 96}, {"c_head_dim": 0},
    {"c_pages": 0}, {"c_kv_heads": 0}, {"c_kv_heads": 65537}, {"c_page_size": 8}, {"c_page_size": 24}, {"c_page_size": 8192}, {"c_page_size": 0},
    {"c_page_size": -16}, {"c_k": None}, {"c_v": None}, {"c_k": 0x10008}, {"c_v": 0x20004}, {"c_k_stride": (2048, 128, 60)},
    {"c_v_stride": (2048, -128, 64)}, {"c_k_stride": (1 << 41, 128, 64)}, {"c_k_stride": (2048, 0, 64)}, {"c_v_stride": (2048, 128, 56)},
    {"c_k_stride": (1 << 40, (1 << 23) + 8, 64)}, {"c_v_stride": (1 << 40, 1 << 23, 64), "c_page_size": 256}, {"c_k_stride": (0, 128, 64)}]
BAD_PAGES = [{"table": None}, {"kv_lens": None}, {"table": 0x1002}, {"q_lens": 0x2002}, {"kv_lens": 0x2001}, {"max_pages": 0}, {"max_pages": 1 << 30},
             {"table_stride": -1}, {"table_stride": 1 << 41}, {"batch": -1}, {"q_len": -1}]


@pytest.mark.parametrize("name", ["tps_cache_append", "tps_cache_read"])
@pytest.mark.parametrize("kw", BAD_CACHE + BAD_PAGES + [
    {"k": None}, {"v": None}, {"k": 0x4008}, {"v": 0x5002}, {"k_stride": (384, 128, 60)}, {"v_stride": (384, -8, 64)}, {"k_stride": (1 << 41, 128, 64)},
    {"batch": 1 << 13, "q_len": 1 << 12}, {"batch": 2 ** 31 - 1, "q_len": 2 ** 31 - 1}, {"batch": 1 << 21, "q_len": 1}, {"reserved": 3}])
def test_row_refusals(name, kw):
    st, msg = _status(name, rows_args(**kw))
    assert st == tp.TP_E_INVAL and msg.startswith(name + ": "), (st, msg)


def test_rows_that_are_written_do_not_overlap():
    kw = {"k_stride": (0, 128, 64)}                 # one sequence's rows for all: may be appended, not read into
    assert _status("tps_cache_read", rows_args(**kw))[0] == tp.TP_E_INVAL
    assert _status("tps_cache_read", rows_args(**{"v_stride": (384, 128, 8)}))[0] == tp.TP_E_INVAL


@pytest.mark.parametrize("kw", BAD_CACHE + BAD_PAGES + [
    {"q": None}, {"out": None}, {"q": 0x4004}, {"out": 0x5008}, {"q_stride": (768, 256, 12)}, {"out_stride": (768, 256, 0)}, {"out_stride": (768, 56, 64)},
    {"q_stride": (768, -256, 64)}, {"heads": 0}, {"heads": 5}, {"heads": 65538}, {"kv_len": -1}, {"kv_len": 1 << 30}, {"sinks": -1},
    {"scale": -1.0}, {"scale": float("nan")}, {"scale": float("inf")}, {"scale": 2e38}, {"work": 0x7010}, {"batch": 1 << 13, "q_len": 1 << 12},
    {"batch": 1 << 21, "q_len": 1}])
def test_attention_refusals(kw):
    st, msg = _status("tps_cache_attention", attention_args(**kw))
    assert st == tp.TP_E_INVAL and msg.startswith("tps_cache_attention: "), (st, msg)


@pytest.mark.parametrize("args,name", [(rows_args, "tps_cache_append"), (attention_args, "tps_cache_attention")])
@pytest.mark.parametrize("kw", [{"c_exps": None}, {"c_exps": 0x30002}, {"c_k_stride": (2048, 128, 72)}, {"c_pages": 1 << 25}, {"c_dtype": tp.TP_BF16}])
def test_refusals_of_8_bit_caches(args, name, kw):
    assert _status(name, args(True, **kw))[0] == tp.TP_E_INVAL


def lora_args(**kw):
    return _set(S.tps_lora_args(x=0x1000, ldx=64, a=0x2000, b=0x3000, a_stride=512, b_stride=256, adapter=0x4000, y=0x5000, ldy=32, dtype=tp.TP_BF16,
                                M=2, N=32, K=64, R=8, adapters=3, act=0), kw)


@pytest.mark.parametrize("kw", [
    {"M": -1}, {"N": 0}, {"K": 0}, {"K": 60}, {"K": (1 << 20) + 8}, {"R": 0}, {"R": 12}, {"R": 136}, {"adapters": 0}, {"act": 3}, {"act": -1}, {"dtype": 2},
    {"dtype": tp.TPS_E4M3}, {"reserved": 1}, {"work": 0x7010}, {"x": None}, {"a": None}, {"b": None}, {"adapter": None}, {"y": None}, {"x": 0x1008},
    {"a": 0x2002}, {"b": 0x3004}, {"adapter": 0x4002}, {"ranks": 0x6001}, {"scales": 0x6002}, {"y": 0x5001}, {"y": 0x5002, "dtype": 0}, {"base": 0x6001},
    {"ldx": 68}, {"ldx": 56}, {"ldx": 1 << 41}, {"ldy": 31}, {"ldy": 1 << 41}, {"base": 0x6000, "ldbase": -32}, {"base": 0x6000, "ldbase": 1 << 41},
    {"base": 0x5000, "ldbase": 64}, {"a_stride": 4}, {"b_stride": -8}, {"a_stride": 1 << 41}, {"M": 1 << 28, "N": 256}, {"M": 2 ** 31 - 1, "N": 2 ** 31 - 1}])
def test_lora_refusals(kw):
    st, msg = _status("tps_lora", lora_args(**kw))
    assert st == tp.TP_E_INVAL and msg.startswith("tps_lora: "), (st, msg)


def test_calls_of_nothing():
    for name in NAMES:
        assert _status(name, None)[0] == tp.TP_E_INVAL
    for name, make in (("tps_cache_append", rows_args), ("tps_cache_read", rows_args), ("tps_cache_attention", attention_args)):
        assert _status(name, make(batch=0)) == (tp.TP_OK, "")
        assert _status(name, make(q_len=0)) == (tp.TP_OK, "")
    assert _status("tps_lora", lora_args(M=0)) == (tp.TP_OK, "")


def test_the_reference_of_8_bit_values():
    v = e4m3_values()
    want = torch.arange(256, dtype=torch.int32).to(torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(v, want, equal_nan=True)
    x = torch.randn(500, 64, generator=torch.Generator().manual_seed(1)).to(torch.bfloat16)
    codes, ex, back = e4m3_rows(x.double().numpy())
    scaled = torch.from_numpy(x.double().numpy() / 2.0 ** (ex[:, None] - 127.0)).float()
    assert float(scaled.abs().max()) <= 448 and bool((scaled.abs().amax(1) > 224).all())
    assert np.array_equal(scaled.to(torch.float8_e4m3fn).view(torch.uint8).numpy() & 127, codes & 127)
    assert (np.abs(back - x.double().numpy()) <= np.maximum(2.0 ** -4 * np.abs(x.double().numpy()), 2.0 ** (ex[:, None] - 137.0))).all()


# ------------------------------------------------------------------ the binding, its calls recorded

class Device(torch.Tensor):
    """A host tensor that says it is on the GPU 1."""

    device = property(lambda self: types.SimpleNamespace(type="cuda", index=1))

    def get_device(self):
        return 1

    def __deepcopy__(self, memo):
        return self.as_subclass(torch.Tensor).clone().as_subclass(Device)


def on(t):
    return t.as_subclass(Device)


@pytest.fixture
def calls(monkeypatch):
    made, entered = [], []
    where = types.SimpleNamespace(type="cuda", index=1)
    monkeypatch.setattr(Device, "device", property(lambda self: where))

    @contextlib.contextmanager
    def device(d):
        entered.append(d)
        yield

    fake = types.SimpleNamespace(bfloat16=torch.bfloat16, float32=torch.float32, int32=torch.int32, cuda=types.SimpleNamespace(device=device))
    call = lambda packed, stream: made.append((packed, stream, list(entered))) or 0       # noqa: E731
    state = types.SimpleNamespace(made=made, entered=entered, stream=0, current=1)
    monkeypatch.setattr(S, "_calls", (fake, lambda d: state.stream, lambda: state.current, call, call, call, call))
    return state


def bf(*shape):
    return on(torch.zeros(*shape, dtype=torch.bfloat16))


def i32(*values):
    return on(torch.tensor(values, dtype=torch.int32))


def a_cache(e4m3=False):
    k, v = (on(torch.zeros(8, 16, 2, 64, dtype=torch.float8_e4m3fn if e4m3 else torch.bfloat16)) for _ in "kv")
    return tp.PagedCache(k, v, on(torch.zeros(8, 2, 2, 16, dtype=torch.uint8)) if e4m3 else None), k, v


def append(cache, **kw):
    a = {"table": on(torch.zeros(3, 5, dtype=torch.int32)), "kv_lens": i32(1, 2, 3), "k": bf(3, 4, 2, 64), "v": bf(3, 4, 2, 64), **kw}
    tp.tps_cache_append(cache, a["table"], a["kv_lens"], a["k"], a["v"], q_lens=a.get("q_lens"), stream=a.get("stream"))


def attend(cache, **kw):
    a = {"table": on(torch.zeros(3, 5, dtype=torch.int32)), "kv_lens": i32(1, 2, 3), "q": bf(3, 4, 6, 64), "out": bf(3, 4, 6, 64), **kw}
    tp.tps_cache_attention(cache, a["table"], a["kv_lens"], a["q"], a["out"], q_lens=a.get("q_lens"), work=a.get("work"), stream=a.get("stream"))


def adapt(_=None, **kw):
    a = {"x": bf(3, 64), "a": bf(2, 8, 64), "b": bf(2, 40, 8), "adapter": i32(0, 1, 1), "out": bf(3, 40), **kw}
    tp.tps_lora(a["x"], a["a"], a["b"], a["adapter"], a["out"], base=a.get("base"), ranks=a.get("ranks"), scales=a.get("scales"),
                work=a.get("work"), stream=a.get("stream"))


def test_what_is_handed_over(calls):
    cache, k, v = a_cache(True)
    append(cache, q_lens=i32(1, 1, 1))
    a = S.tps_cache_rows_args.from_buffer_copy(calls.made[-1][0])
    assert (a.cache.k, a.cache.v, a.cache.dtype, a.cache.pages, a.cache.page_size) == (k.data_ptr(), v.data_ptr(), tp.TPS_E4M3, 8, 16)
    assert (list(a.k_stride), a.batch, a.q_len, a.max_pages, a.table_stride) == ([512, 128, 64], 3, 4, 5, 5)
    attend(cache)
    a = S.tps_cache_attention_args.from_buffer_copy(calls.made[-1][0])
    assert (a.heads, a.kv_len, a.window, a.sinks, a.scale, a.work, a.q_lens) == (6, 80, -1, 0, 0.0, None, None)
    adapt(base=bf(3, 40))
    a = S.tps_lora_args.from_buffer_copy(calls.made[-1][0])
    assert (a.M, a.N, a.K, a.R, a.adapters, a.a_stride, a.b_stride, a.ldbase, a.ranks) == (3, 40, 64, 8, 2, 512, 320, 40, None)


@pytest.mark.parametrize("op", [append, attend, adapt])
@pytest.mark.parametrize("current,stream,entered", [(0, 0, [1]), (0, 4096, []), (1, 0, [])])
def test_the_null_stream_is_the_tensors_devices(op, current, stream, entered, calls):
    calls.current, calls.stream = current, stream
    op(a_cache()[0])
    assert calls.made[-1][1:] == (stream, entered)
    other = types.SimpleNamespace(device=types.SimpleNamespace(index=0), cuda_stream=4096)
    with pytest.raises(ValueError, match="stream of"):
        op(a_cache()[0], stream=other)


@pytest.mark.parametrize("op", [attend, adapt])
def test_scratch_is_the_memory_of_its_tensor(op, calls):
    one = torch.zeros(4096, dtype=torch.uint8)
    for bad in (one[:1].expand(32 << 20), one[::2], one.view(64, 64).t()):
        with pytest.raises(ValueError, match="contiguous"):
            op(a_cache()[0], work=on(bad))
    with pytest.raises(ValueError, match="on device 1"):
        op(a_cache()[0], work=one)
    assert not calls.made
    op(a_cache()[0], work=on(one[256:]))
    a = (S.tps_cache_attention_args if op is attend else S.tps_lora_args).from_buffer_copy(calls.made[0][0])
    assert (a.work, a.work_bytes) == (one.data_ptr() + 256, 4096 - 256)


@pytest.mark.parametrize("kw", [
    {"k": bf(3, 4, 3, 64)}, {"k": bf(3, 4, 2, 128), "v": bf(3, 4, 2, 128)}, {"v": bf(3, 5, 2, 64)}, {"k": on(torch.zeros(3, 4, 2, 64))},
    {"k": bf(3, 4, 2, 128)[..., ::2]}, {"kv_lens": i32(1, 2)}, {"kv_lens": on(torch.zeros(3, dtype=torch.int64))}, {"q_lens": i32(1, 2, 3, 4)},
    {"kv_lens": i32(1, 2, 3, 4, 5, 6)[::2]}, {"table": on(torch.zeros(2, 5, dtype=torch.int32))}, {"table": on(torch.zeros(3, 5))},
    {"table": on(torch.zeros(3, 10, dtype=torch.int32))[:, ::2]}, {"k": torch.zeros(3, 4, 2, 64, dtype=torch.bfloat16)},
    {"kv_lens": torch.zeros(3, dtype=torch.int32)}, {"table": torch.zeros(3, 5, dtype=torch.int32)}])
def test_rows_that_do_not_fit(kw, calls):
    with pytest.raises(ValueError):
        append(a_cache()[0], **kw)
    assert not calls.made


@pytest.mark.parametrize("kw", [
    {"q": bf(3, 4, 6, 128)}, {"out": bf(3, 4, 5, 64)}, {"q": on(torch.zeros(3, 4, 6, 64))}, {"out": bf(3, 4, 64, 6).transpose(2, 3)}, {"q": bf(3, 24, 64)},
    {"kv_lens": i32(1)}, {"q": torch.zeros(3, 4, 6, 64, dtype=torch.bfloat16)}])
def test_queries_that_do_not_fit(kw, calls):
    with pytest.raises(ValueError):
        attend(a_cache()[0], **kw)
    assert not calls.made


@pytest.mark.parametrize("kw", [
    {"x": bf(3, 72)}, {"a": bf(3, 8, 64)}, {"b": bf(2, 40, 16)}, {"b": bf(2, 39, 8)}, {"out": bf(4, 40)}, {"adapter": i32(0, 1)}, {"x": on(torch.zeros(3, 64))},
    {"out": on(torch.zeros(3, 40, dtype=torch.float64))}, {"a": bf(2, 64, 8).transpose(1, 2)}, {"a": bf(2, 8, 128)[..., :64]}, {"b": bf(2, 40, 16)[..., :8]},
    {"out": bf(40, 3).t()}, {"x": bf(64, 3).t()}, {"base": on(torch.zeros(3, 40))}, {"base": bf(3, 41)}, {"base": bf(40, 3).t()}, {"ranks": i32(1)},
    {"scales": on(torch.zeros(2, dtype=torch.bfloat16))}, {"scales": on(torch.zeros(3))}, {"b": torch.zeros(2, 40, 8, dtype=torch.bfloat16)},
    {"adapter": torch.zeros(3, dtype=torch.int32)}, {"x": bf(3, 64, 1)}])
def test_adapters_that_do_not_fit(kw, calls):
    with pytest.raises(ValueError):
        adapt(**kw)
    assert not calls.made


def test_a_cache_keeps_the_memory_that_its_calls_read(calls):
    cache, k, v = a_cache()
    was = k.data_ptr(), v.data_ptr()
    for name, value in (("k", v), ("pages", 99), ("e4m3", True), ("_packed", (0, b""))):
        with pytest.raises(AttributeError):
            setattr(cache, name, value)
    for t in (k, v, cache.k, cache.v):
        t.data = on(torch.ones(8, 16, 2, 64, dtype=torch.bfloat16))
    append(cache)
    a = S.tps_cache_rows_args.from_buffer_copy(calls.made[0][0])
    assert (a.cache.k, a.cache.v) == was == (cache.k.data_ptr(), cache.v.data_ptr())
    for make, shares in ((copy.copy, True), (copy.deepcopy, False)):
        assert (make(cache)._packed == cache._packed) == shares
    for bad in ((k, bf(8, 16, 2, 128), None), (bf(8, 16, 128), bf(8, 16, 128), None), (k, k, on(torch.zeros(8, 2, 2, 16, dtype=torch.uint8))),
                (on(torch.zeros(8, 16, 2, 64)), on(torch.zeros(8, 16, 2, 64)), None), (bf(8, 16, 2, 128)[..., ::2], k, None),
                (torch.zeros(8, 16, 2, 64, dtype=torch.bfloat16),) * 2 + (None,)):
        with pytest.raises(ValueError):
            tp.PagedCache(*bad)
    k8 = on(torch.zeros(8, 16, 2, 64, dtype=torch.uint8))
    for exps in (None, on(torch.zeros(8, 2, 16, 2, dtype=torch.uint8)), on(torch.zeros(8, 2, 2, 16, dtype=torch.int8)),
                 on(torch.zeros(8, 2, 2, 32, dtype=torch.uint8))[..., ::2]):
        with pytest.raises(ValueError):
            tp.PagedCache(k8, k8, exps)
