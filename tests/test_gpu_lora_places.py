"""tps_lora, every kernel: a row's bits do not depend on where it stands, and fp32 results hold every bit of the inner sums."""
import numpy as np
import pytest

from tests.common import log
from tests.test_gpu_lora import Setup
from tests.test_gpu_serve_variants import LORA

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("f32", [False, True])
@pytest.mark.parametrize("i", range(len(LORA)))
def test_a_row_gives_the_same_bits_in_any_place(i, f32):
    # the rows of a call in other orders (as many, so that the plan is the same): neighbours, tiles and the number of an adapter's rows in
    # a tile are others
    import torch
    kernel, m, k, n, r, slots, ids = LORA[i]
    log(f"{kernel} {m} rows, {k} -> {n}, {slots} adapters of {r}, fp32 {f32}")
    s = Setup(1000 + i, m, k, n, r, slots, f32, ids(m, slots), [max(1, r - 3 * (a % 4)) for a in range(slots)])
    x, adapter, base, want = s.x, s.adapter, s.base, s.run("gelu")
    rng = np.random.default_rng(i)
    by_adapter = np.argsort(adapter.cpu().numpy(), kind="stable")
    for perm in (rng.permutation(m), np.arange(m)[::-1].copy(), by_adapter):
        p = torch.from_numpy(perm).to("cuda:0")
        s.x, s.adapter, s.base = x[p].contiguous(), adapter[p].contiguous(), base[p].contiguous()
        assert torch.equal(s.run("gelu"), want[p])


@pytest.mark.parametrize("i", range(len(LORA)))
def test_fp32_results_hold_the_inner_sums_exactly(i):
    # Whole numbers: four values of 8 bits a row times powers of two up to 2^12, so inner sums up to 2^22 that every order of addition gives
    # exactly; an output takes one rank's sum (times 1/2, 1 or 2) and a base of at most 100: 24 bits at most. Two bf16 parts of such a
    # sum, 16 bits, would leave whole units.
    import torch
    kernel, m, k, n, r, slots, ids = LORA[i]
    log(f"{kernel} {m} rows, {k} -> {n}, {slots} adapters of {r}")
    rng = np.random.default_rng(77 + i)
    x = np.zeros((m, k))
    for c in range(4):
        x[np.arange(m), rng.integers(0, k, m)] = rng.integers(-255, 256, m)
    a = 2.0 ** rng.integers(0, 13, (slots, r, k))
    ranks = [max(1, r - 3 * (t % 4)) for t in range(slots)]
    b = np.zeros((slots, n, r))
    for t in range(slots):
        b[t, np.arange(n), rng.integers(0, ranks[t], n)] = 1
    scales = 2.0 ** rng.integers(-1, 2, slots)
    base = rng.integers(-100, 101, (m, n)).astype(np.float64)
    s = Setup(5, 1, 8, 1, 8, 1, True, [0])
    to = lambda v, t: torch.from_numpy(v).to("cuda:0").to(t)                     # noqa: E731
    s.x, s.a, s.b = (to(v, torch.bfloat16) for v in (x, a, b))
    s.base, s.scales, s.ranks = to(base, torch.float32), to(scales, torch.float32), to(np.array(ranks), torch.int32)
    adapter = np.array(ids(m, slots))
    s.adapter = to(adapter, torch.int32)
    y = base.copy()
    for t in range(slots):
        rows = adapter == t
        y[rows] += scales[t] * ((x[rows] @ a[t].T) @ b[t].T)
    for work in (True, False):
        out = s.run(work=work).double().cpu().numpy()
        assert np.array_equal(out, y), (work, float(np.abs(out - y).max()))
