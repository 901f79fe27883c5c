"""The 4-bit format's packing and rounding under AddressSanitizer and UndefinedBehaviorSanitizer, and the binding's check of
a stream against its tensors' device."""
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
