"""What the operators' binding hands to the library (no GPU: the library's calls are recorded, not made)."""
import contextlib
import copy
import types

import pytest

from paper_2306_03622_amd import torpor as T

torch = pytest.importorskip("torch")


class OnDevice1:
    """A host tensor that says it is on device 1."""

    def __init__(self, t):
        self.t = t

    def __getattr__(self, name):
        return getattr(self.t, name)

    def get_device(self):
        return 1


@pytest.fixture
def calls(monkeypatch):
    made = []
    call = lambda packed, stream: made.append(packed) or 0      # noqa: E731
    fake = types.SimpleNamespace(bfloat16=torch.bfloat16, float32=torch.float32, int32=torch.int32,
                                 cuda=types.SimpleNamespace(device=lambda d: contextlib.nullcontext()))
    monkeypatch.setattr(T, "_ops", (fake, lambda d: 4096, lambda: 1, call, call))
    return made


def rows(m, n):
    return OnDevice1(torch.zeros(m, n, dtype=torch.bfloat16))


def linear(work):
    weight = types.SimpleNamespace(_packed=(1, 4096, 4096), out_features=16, in_features=128, group=128)
    T.tpo_linear_w4(rows(3, 128), weight, rows(3, 16), work=work)


def attention(work):
    q = OnDevice1(torch.zeros(2, 3, 4, 64, dtype=torch.bfloat16))
    T.tpo_attention(q, q, q, q, work=work)


@pytest.mark.parametrize("op", [linear, attention])
def test_scratch_is_the_memory_of_its_tensor(op, calls):
    # a tensor that names more bytes than lie behind its address would be written beyond its end
    one = torch.zeros(4096, dtype=torch.uint8)
    for bad in (one[:1].expand(32 << 20), one[::2], one.view(64, 64).t()):
        with pytest.raises(ValueError, match="contiguous"):
            op(OnDevice1(bad))
    with pytest.raises(ValueError, match="on device 1"):
        op(one)
    assert not calls
    op(OnDevice1(one[256:].view(torch.float32)))
    layout, packer = (T.tpo_linear_w4_args, T._LINEAR) if op is linear else (T.tpo_attention_args, T._ATTENTION)
    assert len(calls) == 1 and len(calls[0]) == packer.size
    a = layout.from_buffer_copy(calls[0])
    assert a.work == one.data_ptr() + 256 and a.work_bytes == 4096 - 256


class Device(torch.Tensor):
    """A host tensor whose device is said to be a GPU's."""

    device = property(lambda self: types.SimpleNamespace(type="cuda", index=1))

    def __deepcopy__(self, memo):
        return self.as_subclass(torch.Tensor).clone().as_subclass(Device)


def test_a_weight_keeps_the_memory_that_its_calls_read(calls):
    codes, scales = torch.zeros(2048, dtype=torch.uint8), torch.zeros(32, dtype=torch.bfloat16)
    was = codes.data_ptr(), scales.data_ptr()
    mine = codes.as_subclass(Device), scales.as_subclass(Device)
    w = T.W4Weight(*mine, 32, 128, 128)
    other = torch.ones(2048, dtype=torch.uint8), torch.ones(32, dtype=torch.bfloat16)
    for name, value in (("codes", other[0]), ("scales", other[1]), ("out_features", 4096), ("in_features", 256), ("group", 32),
                        ("device", None), ("_packed", (0, 0, 0))):
        with pytest.raises(AttributeError):
            setattr(w, name, value)
    for t, o in zip((*mine, w.codes, w.scales, codes, scales), (*other, *other, *other)):
        t.data = o                       # gives the tensor object other memory; the weight's stays, and so does its own object
    T.tpo_linear_w4(rows(3, 128), w, rows(3, 32))
    a = T.tpo_linear_w4_args.from_buffer_copy(calls[0])
    assert (a.wq, a.scales) == was and (a.N, a.K, a.group) == (32, 128, 128)
    assert (w.codes.data_ptr(), w.scales.data_ptr()) == was
    assert w.codes.numel() == 2048 and not bool(w.codes.any())      # the memory is still there, as it was
    for make, shares in ((copy.copy, True), (copy.deepcopy, False)):
        c = make(w)
        assert (c._packed == w._packed) == shares and c._packed[1] == c.codes.data_ptr() and c.out_features == 32
    w._codes.fill_(3)
    assert bool((w.codes == 3).all())
