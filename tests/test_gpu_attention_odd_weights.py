"""tpo_attention where infinities and NaN meet weights that round to zero, with the keys split over workgroups and not."""
import pytest

from tests.common import log
from tests.test_gpu_attention_masked import make, run

pytestmark = pytest.mark.gpu

# (dim, heads, key/value heads, queries, keys): few rows over many keys are split where there is scratch
SHAPES = [(64, 8, 1, 1, 9000), (128, 8, 2, 1, 20000), (128, 32, 8, 1, 40000), (64, 4, 4, 5, 3000), (128, 4, 2, 200, 700)]


@pytest.mark.parametrize("d,h,hk,nq,nk", SHAPES)
@pytest.mark.parametrize("work", [True, False])
def test_an_infinite_value_of_next_to_no_weight_shows(d, h, hk, nq, nk, work):
    # the last hundred keys outweigh the others by exp(800): those weigh nothing that fp32 holds, but more than nothing
    log(f"{nq} over {nk}, {h} / {hk} heads of {d}, scratch {work}")
    q, k, v = make(d + nk, 1, nq, nk, h, hk, d)
    q.fill_(8.0)
    k.zero_()
    k[:, nk - 100:] = 800 / (8 * d ** 0.5)
    for value, key in ((float("inf"), 3), (float("-inf"), nk // 2), (float("nan"), nk - 200), (float("inf"), nk - 1)):
        clean = run(q, k, v, work=work)
        v2 = v.clone()
        v2[0, key, hk - 1, 5] = value
        got, want = run(q, k, v2, work=work), clean.clone()
        want[:, :, h - h // hk:, 5] = value
        assert bool(((got == want) | (got.isnan() & want.isnan())).all()), (value, key)
