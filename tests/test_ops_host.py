"""The operators' host side (no GPU): exported symbols, struct layouts, the 4-bit format, quantisation, and every
refusal of invalid arguments, which comes before any launch."""
import ctypes
import os
import re
import shutil
import subprocess

import numpy as np
import pytest

import paper_2306_03622_amd as tp
import synth
from paper_2306_03622_amd import torpor as T
from tests.ops_common import w4_matrix, w4_plain

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_library_exports_the_operators_header():
    src = open(os.path.join(ROOT, "include", "torpor_ops.h")).read()
    declared = set(re.findall(r"^TP_API\s+[\w\s\*]+?\b(tpo_\w+)\s*\(", src, re.M))
    assert declared == {"tpo_w4_bytes", "tpo_w4_pack", "tpo_w4_quantize", "tpo_linear_w4", "tpo_attention"}
    out = subprocess.run(["nm", "-D", "--defined-only", T.LIB_PATH], capture_output=True, text=True).stdout
    assert set(re.findall(r" T (tpo_\w+)", out)) == declared
    host = subprocess.run(["nm", "-D", "--defined-only", T.HOST_LIB_PATH], capture_output=True, text=True).stdout
    assert set(re.findall(r" T (tpo_\w+)", host)) == {n for n in declared if n.startswith("tpo_w4_")}
    assert int(re.search(r"TPO_WORK_BYTES \((\d+)u << 20\)", src).group(1)) << 20 == tp.TPO_WORK_BYTES


@pytest.mark.parametrize("name", ["tpo_linear_w4_args", "tpo_attention_args"])
def test_ctypes_layout_matches_the_header(name, tmp_path):
    cc = shutil.which("gcc") or shutil.which("cc")
    if not cc:
        pytest.skip("no C compiler")
    cls = getattr(T, name)
    src = ["#include <stdio.h>", "#include <stddef.h>", '#include "torpor_ops.h"', "int main(void) {",
           f'  printf("size %zu\\n", sizeof({name}));']
    src += [f'  printf("{f} %zu\\n", offsetof({name}, {f}));' for f, _ in cls._fields_] + ["  return 0;", "}"]
    (tmp_path / "l.c").write_text("\n".join(src) + "\n")
    subprocess.run([cc, "-std=c11", "-I", os.path.join(ROOT, "include"), str(tmp_path / "l.c"), "-o", str(tmp_path / "l")],
                   check=True)
    got = dict(l.split() for l in subprocess.run([str(tmp_path / "l")], check=True, capture_output=True, text=True).stdout.splitlines())
    assert int(got.pop("size")) == ctypes.sizeof(cls)
    assert {f: int(v) for f, v in got.items()} == {f: getattr(cls, f).offset for f, _ in cls._fields_}


def test_packed_arguments_have_the_structs_layout():
    for packer, cls, values in ((T._LINEAR, T.tpo_linear_w4_args, list(range(1, 18))),
                                (T._ATTENTION, T.tpo_attention_args, [*range(1, 29), 0.5, 30, 31])):
        assert packer.size == ctypes.sizeof(cls)
        a, got = cls.from_buffer_copy(packer.pack(*values)), []
        for name, _ in cls._fields_:
            v = getattr(a, name)
            got += list(v) if hasattr(v, "__len__") else [v]
        assert got == values


def unblock(codes, scales, n, k, group):
    """The matrix of blocked codes and scales, element by element from the format's description."""
    kb, ng = (k + 127) // 128, (k + 127) // 128 * (128 // group)
    w = np.zeros((n, k))
    s = synth.bf16_to_f32(scales).astype(np.float64)
    for row in range(n):
        for col in range(k):
            t, q, c = col % 128 // 32, col % 32 // 8, col % 8
            word = ((row // 16) * kb + col // 128) * 256 + 4 * (16 * q + row % 16) + t
            bit = 4 * (c // 2) + 16 * (c % 2)
            code = (codes[4 * word + bit // 8] >> (bit % 8)) & 15
            w[row, col] = (int(code) - 8) * s[((row // 16) * ng + col // group) * 16 + row % 16]
    return w


@pytest.mark.parametrize("n,k,group", [(1, 32, 32), (16, 128, 128), (17, 96, 32), (40, 192, 64), (33, 256, 128), (5, 160, 32)])
@pytest.mark.parametrize("which", ["lib", "host_lib"])
def test_blocked_order(n, k, group, which):
    L = getattr(tp, which)()
    rng = np.random.default_rng(n * 1000 + k)
    codes, bits, w = w4_plain(rng, n, k, group)
    assert np.array_equal(w4_matrix(codes, bits, group), w)
    bc, bs = tp.tpo_w4_pack(codes, bits, group, L=L)
    assert (bc.nbytes, bs.nbytes) == tp.tpo_w4_bytes(n, k, group, L=L)
    assert bc.nbytes == (n + 15) // 16 * ((k + 127) // 128) * 1024
    assert np.array_equal(unblock(bc, bs, n, k, group), w)
    # what stands for no element is padding: code 8 everywhere, scale 0
    full_n, full_k = (n + 15) // 16 * 16, (k + 127) // 128 * 128
    full = unblock(bc, np.full_like(bs, 0x3F80), full_n, full_k, group)
    full[:n, :k] = 0
    assert not full.any()
    assert np.count_nonzero(bs) == np.count_nonzero(bits)


def test_quantisation_rounds_to_the_nearest_of_fifteen():
    rng = np.random.default_rng(5)
    w = rng.standard_normal((24, 256)).astype(np.float32)
    w[3, 32:64] = 0
    w[4, :32] = 1e-42          # a scale below the smallest bf16: the group becomes zero
    for group in (32, 64, 128):
        codes, bits = tp.tpo_w4_quantize(w, group, L=tp.host_lib())
        back = w4_matrix(codes, bits, group)
        s = np.repeat(synth.bf16_to_f32(bits).astype(np.float64), group, axis=1)
        both = np.stack([codes & 15, codes >> 4])
        assert both.min() >= 1 and both.max() <= 15
        # half a step, and at the end of the range what the scale's own rounding (2^-8 of it, times 7) leaves
        assert (np.abs(back - w) <= s * (0.5 + 7 * 2.0 ** -8) + 1e-40).all()
        top = np.abs(w).reshape(24, -1, group).max(axis=2) / 7
        assert np.array_equal(bits, synth.bf16_round(top.astype(np.float32)).reshape(bits.shape))
    assert not w4_matrix(*tp.tpo_w4_quantize(np.zeros((2, 64), np.float32), 32, L=tp.host_lib()), 32).any()


def test_quantisation_refuses_what_has_no_scale():
    for bad in (np.inf, -np.inf, np.nan):
        w = np.zeros((2, 64), dtype=np.float32)
        w[1, 40] = bad
        with pytest.raises(tp.TorporError):
            tp.tpo_w4_quantize(w, 32, L=tp.host_lib())


@pytest.mark.parametrize("n,k,group", [(0, 32, 32), (1, 0, 32), (1, 48, 32), (1, 64, 128), (1, 64, 16), (1, 64, 0), (-1, 32, 32),
                                       ((1 << 24) + 1, 32, 32), (1, (1 << 20) + 32, 32)])
def test_shapes_that_are_refused(n, k, group):
    for L in (tp.lib(), tp.host_lib()):
        with pytest.raises(tp.TorporError) as e:
            tp.tpo_w4_bytes(n, k, group, L=L)
        assert e.value.status == tp.TP_E_INVAL


def _status(name, args):
    L = tp.lib()
    st = getattr(L, name)(None if args is None else ctypes.byref(args), None)
    return st, L.tp_last_error().decode()


# (addresses below are never read: every call here is refused before a launch)
def linear_args(**kw):
    a = T.tpo_linear_w4_args(x=0x1000, ldx=64, wq=0x2000, scales=0x3000, y=0x4000, ldy=32, y_dtype=tp.TP_BF16, M=2, N=32, K=64,
                             group=32, act=0)
    for k, v in kw.items():
        setattr(a, k, v)
    return a


@pytest.mark.parametrize("kw", [
    {"M": -1}, {"N": 0}, {"K": 0}, {"K": 48}, {"group": 16}, {"group": 128}, {"act": 3}, {"act": -1}, {"y_dtype": 2}, {"x": None},
    {"wq": None}, {"scales": None}, {"y": None}, {"x": 0x1008}, {"ldx": 68}, {"ldx": 56}, {"ldy": 31}, {"wq": 0x2008}, {"scales": 0x3002},
    {"y": 0x4001}, {"y": 0x4002, "y_dtype": 0}, {"bias": 0x5001}, {"res": 0x6001, "ldr": 32}, {"res": 0x6000, "ldr": 31},
    {"work": 0x7010}, {"res": 0x4000, "ldr": 40}, {"res": 0x4000, "ldr": 32, "y_dtype": 0}, {"ldx": 1 << 41}, {"ldy": 1 << 41}])
def test_linear_refusals(kw):
    st, msg = _status("tpo_linear_w4", linear_args(**kw))
    assert st == tp.TP_E_INVAL and msg.startswith("tpo_linear_w4: "), (st, msg)


def attention_args(**kw):
    a = T.tpo_attention_args(q=0x1000, k=0x2000, v=0x3000, out=0x4000, batch=2, heads=4, kv_heads=2, head_dim=64, q_len=8, kv_len=16,
                             window_left=-1, window_right=-1)
    for f, h, n in (("q_stride", 4, 8), ("k_stride", 2, 16), ("v_stride", 2, 16), ("out_stride", 4, 8)):
        for i, s in enumerate((n * h * 64, h * 64, 64)):
            getattr(a, f)[i] = s
    for k, v in kw.items():
        if isinstance(v, tuple):
            for i, s in enumerate(v):
                getattr(a, k)[i] = s
        else:
            setattr(a, k, v)
    return a


@pytest.mark.parametrize("kw", [
    {"batch": -1}, {"q_len": -1}, {"kv_len": -1}, {"q_len": 1 << 30}, {"kv_len": 1 << 30}, {"heads": 0}, {"kv_heads": 0}, {"kv_heads": 3},
    {"heads": 1 << 17}, {"head_dim": 80}, {"causal": 2}, {"sinks": -1}, {"scale": -1.0}, {"scale": float("nan")}, {"scale": float("inf")},
    {"work": 0x80}, {"q": None}, {"k": None}, {"v": None}, {"out": None}, {"q": 0x1008}, {"k": 0x2002}, {"v": 0x3008}, {"out": 0x4008},
    {"q_lens": 0x5002}, {"kv_lens": 0x5001}, {"q_stride": (-8, 256, 64)}, {"k_stride": (2048, 130, 64)}, {"v_stride": (2048, 128, 1 << 41)}, {"k_stride": (2048, (1 << 23) + 8, 64)}, {"v_stride": (2048, 1 << 24, 64)},
    {"out_stride": (2048, 256, 56)}, {"out_stride": (0, 256, 64)}, {"batch": 1 << 20, "q_len": 1 << 10},
    {"batch": 1 << 21, "q_len": 1}])
def test_attention_refusals(kw):
    st, msg = _status("tpo_attention", attention_args(**kw))
    assert st == tp.TP_E_INVAL and msg.startswith("tpo_attention: "), (st, msg)


def test_calls_of_nothing_succeed_without_a_device():
    for name, a in (("tpo_linear_w4", linear_args(M=0)), ("tpo_attention", attention_args(batch=0)),
                    ("tpo_attention", attention_args(q_len=0))):
        assert _status(name, a) == (tp.TP_OK, "")
    for name in ("tpo_linear_w4", "tpo_attention"):
        assert _status(name, None)[0] == tp.TP_E_INVAL


def test_binding_refuses_tensors_that_do_not_belong_together():
    torch = pytest.importorskip("torch")
    with pytest.raises(ValueError, match="belong together"):
        tp.tpo_w4_pack(np.zeros((4, 32), np.uint8), np.zeros((4, 3), np.uint16), 32)
    c, s = torch.zeros(1024, dtype=torch.uint8), torch.zeros(16, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="on cpu"):
        tp.W4Weight(c, s, 16, 128, 128)
    with pytest.raises(ValueError, match="need"):
        tp.W4Weight(c, s, 17, 128, 128)
    with pytest.raises(ValueError, match="uint8"):
        tp.W4Weight(c.to(torch.int32), s, 16, 128, 128)
    q = torch.zeros(1, 4, 2, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="on cpu"):
        tp.tpo_attention(q, q, q, q.clone())
    with pytest.raises(ValueError):
        tp.tpo_attention(q, q[..., :32], q[..., :32], q.clone())


def test_the_gpu_shapes_reach_every_variant(tmp_path):
    from tests.test_gpu_linear_w4 import SHAPES
    cxx = shutil.which("g++")
    if not cxx:
        pytest.skip("no C++ compiler")
    (tmp_path / "d.cpp").write_text('#include <cstdio>\n#include "w4_plan.hpp"\nusing namespace tp::k;\nint main() {\n  long m, n, k;\n  int g;\n'
                                    '  std::printf("%d\\n", (int)W4_VARIANTS);\n  while (std::scanf("%ld %ld %ld %d", &m, &n, &k, &g) == 4) '
                                    'std::printf("%d\\n", w4_plan(m, n, k, g));\n}\n')
    subprocess.run([cxx, "-std=c++17", "-I", os.path.join(ROOT, "paper_2306_03622_amd", "csrc", "kernels"), str(tmp_path / "d.cpp"),
                    "-o", str(tmp_path / "d")], check=True)
    more = [(1, 1, 32, 32), (10 ** 7, 16, 32, 32), (3 * 10 ** 6, 1, 1024, 64)]
    out = subprocess.run([str(tmp_path / "d")], input="\n".join(" ".join(map(str, s)) for s in [*SHAPES, *more]), check=True,
                         capture_output=True, text=True).stdout.split()
    n, plans = int(out[0]), [int(v) for v in out[1:]]
    assert set(plans[:len(SHAPES)]) == set(range(n))
    # the kernels of few rows put row tiles into a grid dimension of 65535: millions of rows are for the others
    assert all(p > 2 for p in plans[-2:])
