"""tpo_linear_w4 against the product in 64 bits: exactly where every sum is exact, else within the rounding's bound."""
import numpy as np
import pytest

import synth
from tests.common import log, to_device
from tests.ops_common import act, w4_plain, w4_tolerance

pytestmark = pytest.mark.gpu


def weight(codes, bits, group):
    import paper_2306_03622_amd as tp
    return tp.W4Weight.from_plain(codes, bits, group, device="cuda:0")


def bf_tensor(x):
    import torch
    return to_device(synth.bf16_round(np.asarray(x, dtype=np.float32)).reshape(x.shape)).view(torch.bfloat16)


def scratch():
    import paper_2306_03622_amd as tp
    import torch
    return torch.empty(tp.TPO_WORK_BYTES, dtype=torch.uint8, device="cuda:0").fill_(255)


def run(x, w, f32=False, bias=None, res=None, name="none", work=None, stream=None, pad=0):
    """One call; rows `pad` elements apart more than they are long, which must stay as they were."""
    import paper_2306_03622_amd as tp
    import torch
    m, n = x.shape[0], w.out_features
    base = torch.full((m, n + pad), 7.0, dtype=torch.float32 if f32 else torch.bfloat16, device="cuda:0")
    tp.tpo_linear_w4(x, w, base[:, :n], bias=bias, res=res, act=name, work=work, stream=stream)
    torch.cuda.synchronize()
    assert pad == 0 or bool((base[:, n:] == 7).all())
    return base[:, :n].double().cpu().numpy()


# rows: one, around whole 16s and tiles; features and columns that fill no block; the three groups; every kernel variant
# (test_ops_host.py checks that)
SHAPES = [(1, 16, 128, 128), (1, 1, 32, 32), (2, 17, 96, 32), (7, 40, 192, 64), (8, 256, 512, 128), (15, 33, 160, 32),
          (16, 48, 384, 128), (17, 100, 64, 64), (31, 130, 1024, 64), (32, 64, 256, 32), (33, 96, 128, 128), (48, 70, 640, 128),
          (64, 256, 2048, 64), (65, 257, 224, 32), (100, 1000, 2048, 64), (127, 72, 352, 32), (130, 520, 896, 128),
          (200, 768, 768, 32), (257, 129, 512, 64), (513, 300, 1152, 128), (700, 1024, 320, 64), (1100, 600, 416, 32),
          (2049, 1040, 768, 128), (67, 2100, 640, 64), (20, 9000, 352, 32), (250, 1000, 1152, 64), (67, 1000, 4096, 32),
          (130, 500, 4096, 128), (333, 1000, 4096, 128), (333, 4100, 1088, 64), (513, 4100, 1152, 32), (1025, 2100, 1152, 128),
          (1300, 2300, 2048, 64), (1025, 4100, 2048, 128), (1300, 4100, 1088, 32)]


@pytest.mark.parametrize("m,n,k,group", SHAPES)
def test_exact_sums(m, n, k, group):
    # small whole inputs, codes and powers of two: every product, partial sum and scaled sum is a multiple of 1/8
    # below 2^24 / 8 (|x| <= 3, at most 31 * 3 * 2048 in a group's partial sum), so fp32 holds the result exactly
    rng = np.random.default_rng(m * 7919 + n * 31 + k)
    log(f"exact {m} x {n} x {k}, groups of {group}")
    codes, bits, w = w4_plain(rng, n, k, group, exact=True)
    x = rng.integers(-3, 4, size=(m, k)).astype(np.float64)
    got = run(bf_tensor(x), weight(codes, bits, group), f32=True, work=scratch())
    assert np.array_equal(got, x @ w.T)


@pytest.mark.parametrize("m,n,k,group", SHAPES)
@pytest.mark.parametrize("f32", [False, True])
def test_results(m, n, k, group, f32):
    rng = np.random.default_rng(m * 7919 + n * 31 + k + 1)
    log(f"{m} x {n} x {k}, groups of {group}, fp32 {f32}")
    codes, bits, w = w4_plain(rng, n, k, group)
    x = synth.bf16_to_f32(synth.bf16_round(rng.standard_normal((m, k)).astype(np.float32))).astype(np.float64).reshape(m, k)
    b = rng.standard_normal(n).astype(np.float32) * 0.5
    r = rng.standard_normal((m, n)).astype(np.float32)
    bt, rt = bf_tensor(b), bf_tensor(r)
    bias, res = bt.double().cpu().numpy(), rt.double().cpu().numpy()
    wt, xt = weight(codes, bits, group), bf_tensor(x)
    for name, with_bias, with_res in (("none", False, False), ("gelu", True, False), ("relu", True, True)):
        want = x @ w.T + (bias if with_bias else 0) + (res if with_res else 0)
        tol = w4_tolerance(x, w, want, f32)
        got = run(xt, wt, f32=f32, bias=bt if with_bias else None, res=rt if with_res else None, name=name, work=scratch())
        # 4 more fp32 roundings: bias, residual, their sums
        off = np.abs(got - act(want, name)) - tol - 2.0 ** -22 * (np.abs(want) + np.abs(res if with_res else 0))
        assert off.max() <= 0, (name, float(off.max()), np.unravel_index(off.argmax(), off.shape))


@pytest.mark.parametrize("m", [1, 20, 70, 300])
def test_strides_alignment_and_scratch(m):
    import torch
    rng = np.random.default_rng(m)
    n, k, group = 131, 256, 64
    codes, bits, w = w4_plain(rng, n, k, group, exact=True)
    x = rng.integers(-3, 4, size=(m, k)).astype(np.float64)
    want, wt = x @ w.T, weight(codes, bits, group)
    wide = torch.full((m, k + 24), float("nan"), dtype=torch.bfloat16, device="cuda:0")
    wide[:, 8:8 + k] = bf_tensor(x)
    for work in (None, scratch(), scratch()[:4096]):
        for pad in (0, 1, 2, 5):
            assert np.array_equal(run(wide[:, 8:8 + k], wt, f32=True, pad=pad, work=work), want)
    # outputs, bias and residual at odd elements
    base = torch.zeros(m * n + 1, dtype=torch.float32, device="cuda:0")
    import paper_2306_03622_amd as tp
    bias = torch.arange(n + 1, device="cuda:0").to(torch.bfloat16) % 8
    res = torch.ones(m * n + 1, dtype=torch.bfloat16, device="cuda:0")
    tp.tpo_linear_w4(wide[:, 8:8 + k], wt, base[1:].view(m, n), bias=bias[1:], res=res[1:].view(m, n))
    assert np.array_equal(base[1:].view(m, n).double().cpu().numpy(), want + bias[1:].double().cpu().numpy() + 1)
    # the residual may be the output
    y = torch.full((m, n), 3.0, dtype=torch.bfloat16, device="cuda:0")
    tp.tpo_linear_w4(wide[:, 8:8 + k], wt, y, res=y)
    assert np.array_equal(y.double().cpu().numpy(), torch.tensor(want + 3).to(torch.bfloat16).double().numpy())


@pytest.mark.parametrize("m", [3, 40, 260])
def test_rows_are_their_own(m):
    # an infinite or NaN input touches its own row alone; a row's result does not depend on its neighbours
    import torch
    rng = np.random.default_rng(m + 50)
    n, k, group = 96, 384, 128
    codes, bits, _ = w4_plain(rng, n, k, group)
    wt, x = weight(codes, bits, group), bf_tensor(rng.standard_normal((m, k)))
    clean = run(x, wt, f32=True, work=scratch())
    dirty = x.clone()
    dirty[1, 5], dirty[2, 7] = float("inf"), float("nan")
    got = run(dirty, wt, f32=True, work=scratch())
    assert np.isnan(got[1:3]).all()
    keep = np.arange(m) != 1
    keep[2] = False
    assert np.array_equal(got[keep], clean[keep])


def test_streams_and_graphs():
    import paper_2306_03622_amd as tp
    import torch
    rng = np.random.default_rng(3)
    n, k, group = 272, 1024, 128
    codes, bits, _ = w4_plain(rng, n, k, group)
    wt = weight(codes, bits, group)
    for m in (1, 24, 100, 600):
        xs = [bf_tensor(rng.standard_normal((m, k))) for _ in range(3)]
        want = [run(x, wt, f32=True, work=scratch()) for x in xs]
        side = torch.cuda.Stream(device="cuda:0")
        assert np.array_equal(run(xs[0], wt, f32=True, work=scratch(), stream=side), want[0])
        x, work = xs[0].clone(), scratch()
        out = torch.zeros(m, n, dtype=torch.float32, device="cuda:0")
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            tp.tpo_linear_w4(x, wt, out, work=work)
        for i in (0, 1, 2, 0):
            x.copy_(xs[i])
            out.fill_(-1)
            run(xs[2], wt, f32=True, work=work)           # an eager call between the replays
            g.replay()
            torch.cuda.synchronize()
            assert np.array_equal(out.double().cpu().numpy(), want[i])


def test_quantised_weights_end_to_end():
    # what a program does with fp32 weights: quantise, lay out once, multiply
    import paper_2306_03622_amd as tp
    from tests.ops_common import w4_matrix
    rng = np.random.default_rng(9)
    w = (rng.standard_normal((200, 512)) / 16).astype(np.float32)
    codes, bits = tp.tpo_w4_quantize(w, 64)
    x = bf_tensor(rng.standard_normal((5, 512)))
    xd, wd = x.double().cpu().numpy(), w4_matrix(codes, bits, 64)
    got = run(x, weight(codes, bits, 64), f32=True)
    assert (np.abs(got - xd @ wd.T) <= w4_tolerance(xd, wd, xd @ wd.T, True)).all()
