"""Every kernel of tpo_linear_w4 with every group size that test_gpu_linear_w4.py leaves out: each pair is code of its own (the scales
lie, load and apply otherwise). test_w4_plan.py checks that the two files together reach all pairs."""
import pytest

import tests.test_gpu_linear_w4 as w4

pytestmark = pytest.mark.gpu

# rows and features that are no multiples of the tiles, columns that end inside a block
SHAPES = [(50, 2100, 288, 32), (50, 4100, 320, 64), (50, 4100, 256, 128), (50, 4100, 4128, 32), (50, 4100, 4160, 64),
          (200, 4100, 288, 32), (200, 4100, 256, 128), (200, 5003, 4160, 64), (2050, 1500, 2048, 128), (3001, 2100, 2080, 32),
          (1030, 4100, 2112, 64)]


@pytest.mark.parametrize("m,n,k,group", SHAPES)
def test_exact_sums(m, n, k, group):
    w4.test_exact_sums(m, n, k, group)


@pytest.mark.parametrize("m,n,k,group", SHAPES)
@pytest.mark.parametrize("f32", [False, True])
def test_results(m, n, k, group, f32):
    w4.test_results(m, n, k, group, f32)
