"""The 4-bit format's packing and rounding under AddressSanitizer and UndefinedBehaviorSanitizer, and the binding's streams and
devices."""
import contextlib
import os
import subprocess
import types

import pytest

import paper_2306_03622_amd.build as tp_build
from paper_2306_03622_amd import torpor as T

HERE = os.path.dirname(os.path.abspath(__file__))
INCLUDE = os.path.join(os.path.dirname(HERE), "include")


@pytest.mark.slow
def test_packing_and_rounding_stay_inside_their_buffers(tmp_path):
    lib = tp_build.build_host(str(tmp_path / "libtorpor_host_san.so"), sanitize=True)
    exe = str(tmp_path / "driver")
    r = subprocess.run(["g++", "-O1", "-std=c++17", *tp_build.SANITIZE, f"-I{INCLUDE}",
                        os.path.join(HERE, "ops_sanitize_driver.cpp"), lib, f"-Wl,-rpath,{tmp_path}", "-o", exe],
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    r = subprocess.run([exe], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stdout + r.stderr[-4000:]


def test_a_stream_of_another_device_is_refused():
    stream = types.SimpleNamespace(device=types.SimpleNamespace(index=1), cuda_stream=4096)
    with pytest.raises(ValueError, match="stream of"):
        T._stream_of(0, stream)
    assert T._stream_of(1, stream) == 4096
    assert T._stream_of(0, 4096) == 4096              # a raw handle carries no device: its own is asked at the C entry


class _FakeTensor:
    """What the binding asks of a contiguous tensor, on device 1."""

    def __init__(self, dtype, *shape):
        self.dtype, self.shape, self.device = dtype, shape, "device 1"

    def stride(self, d=None):
        strides = [1]
        for n in reversed(self.shape[1:]):
            strides.insert(0, strides[0] * n)
        return tuple(strides) if d is None else strides[d]

    def dim(self):
        return len(self.shape)

    def get_device(self):
        return 1

    def data_ptr(self):
        return 4096


@pytest.mark.parametrize("current,stream,entered", [(0, 0, [1]), (0, 4096, []), (1, 0, [])])
def test_the_null_stream_is_the_tensors_devices(monkeypatch, current, stream, entered):
    # the tensors are on device 1: the null stream alone says nothing of the device
    import torch
    seen, calls = [], []

    @contextlib.contextmanager
    def device(d):
        seen.append(d)
        yield

    fake = types.SimpleNamespace(bfloat16=torch.bfloat16, float32=torch.float32, cuda=types.SimpleNamespace(device=device))
    call = lambda packed, s: calls.append((s, list(seen))) or 0
    monkeypatch.setattr(T, "_ops", (fake, lambda d: stream, lambda: current, call, call))
    q = _FakeTensor(torch.bfloat16, 2, 3, 4, 64)
    T.tpo_attention(q, q, q, q)
    assert calls == [(stream, entered)]
    seen.clear()
    weight = types.SimpleNamespace(_packed=(1, 4096, 4096), out_features=16, in_features=128, group=128)
    T.tpo_linear_w4(_FakeTensor(torch.bfloat16, 3, 128), weight, _FakeTensor(torch.bfloat16, 3, 16), stream=stream)
    assert calls[1] == (stream, entered)
