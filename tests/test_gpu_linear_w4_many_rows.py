"""tpo_linear_w4 with more rows than the second dimension of a grid holds in sixteens."""
import numpy as np
import pytest

from tests.common import log
from tests.ops_common import w4_plain
from tests.test_gpu_linear_w4 import weight

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n,k,group", [(16, 512, 128), (3, 416, 32), (16, 32, 32)])
def test_exact_sums(n, k, group):
    import torch
    import paper_2306_03622_amd as tp
    m = 65535 * 16 + 1
    log(f"{m} x {n} x {k}, groups of {group}")
    codes, bits, w = w4_plain(np.random.default_rng(k), n, k, group, exact=True)
    g = torch.Generator(device="cuda:0")
    g.manual_seed(k)
    x = torch.randint(-3, 4, (m, k), generator=g, device="cuda:0", dtype=torch.int8).to(torch.bfloat16)
    out = torch.full((m, n), 7.0, dtype=torch.float32, device="cuda:0")
    tp.tpo_linear_w4(x, weight(codes, bits, group), out)
    # every product and sum is a multiple of 1/8 below 2^24 / 8: exact in fp32, in whatever order
    want = x.float() @ torch.tensor(w.T.copy(), dtype=torch.float32, device="cuda:0")
    assert bool((out == want).all())
