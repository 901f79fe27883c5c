"""tpo_linear_w4 on inputs that are infinite or not a number, and on zeros, with each activation, and a model that inherits it."""
import numpy as np
import pytest

import synth
from tests.common import infer, log, make_runtime
from tests.ops_common import act, w4_plain
from tests.test_gpu_linear_w4 import bf_tensor, run, weight

pytestmark = pytest.mark.gpu

# rows, features: few rows and tiles; features in whole vectors, and not
SHAPES = [(3, 96), (20, 33), (130, 96), (300, 131), (1100, 640)]


@pytest.mark.parametrize("m,n", SHAPES)
@pytest.mark.parametrize("name", ["none", "relu", "gelu"])
@pytest.mark.parametrize("f32", [False, True])
def test_odd_rows_are_not_numbers_and_stay_alone(m, n, name, f32):
    log(f"{m} x {n}, {name}, fp32 {f32}")
    rng = np.random.default_rng(m * 31 + n)
    codes, bits, _ = w4_plain(rng, n, 256, 64)
    wt, x = weight(codes, bits, 64), bf_tensor(rng.standard_normal((m, 256)))
    bias, res = bf_tensor(rng.standard_normal(n)), bf_tensor(rng.standard_normal((m, n)))
    for kw in ({}, {"bias": bias, "res": res}):
        clean = run(x, wt, f32=f32, name=name, **kw)
        dirty = x.clone()
        dirty[0, 7], dirty[1, 200], dirty[m - 1, 0] = float("inf"), float("nan"), float("-inf")
        got = run(dirty, wt, f32=f32, name=name, **kw)
        assert np.isnan(got[[0, 1, m - 1]]).all()
        keep = np.ones(m, dtype=bool)
        keep[[0, 1, m - 1]] = False
        assert np.array_equal(got[keep], clean[keep])


@pytest.mark.parametrize("m,n", SHAPES)
def test_relu_of_exact_sums(m, n):
    # sums that fp32 holds exactly (test_gpu_linear_w4.py), a third of the rows zeros: nothing but zeros and the positive sums
    rng = np.random.default_rng(m + 7 * n)
    codes, bits, w = w4_plain(rng, n, 256, 64, exact=True)
    x = rng.integers(-3, 4, size=(m, 256)).astype(np.float64)
    x[::3] = 0
    got = run(bf_tensor(x), weight(codes, bits, 64), f32=True, name="relu")
    assert np.array_equal(got, act(x @ w.T, "relu")) and not np.signbit(got).any()


def test_a_model_shows_an_infinite_input():
    m = synth.quantised(synth.mlp(3, 256, "bf16", "relu", 21), 64)
    x = synth.mlp_input(5, 256, m.dtype, 77)
    rt, (mid,) = make_runtime([m], batch_max=5)
    clean = infer(rt, mid, m, x)
    x[2, 9] = 0x7F80
    got = infer(rt, mid, m, x)
    rt.close()
    assert np.isnan(got[2]).all() and np.array_equal(got[[0, 1, 3, 4]], clean[[0, 1, 3, 4]])
