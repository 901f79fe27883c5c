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


@pytest.mark.parametrize("d,h,hk,nq,nk", SHAPES)
@pytest.mark.parametrize("work", [True, False])
def test_scores_of_minus_infinity(d, h, hk, nq, nk, work):
    # all of them: zeros, whatever the values hold; all but one key's: that key's value, and infinities that any seen key holds
    log(f"{nq} over {nk}, {h} / {hk} heads of {d}, scratch {work}")
    q, k, v = make(d + nk, 1, nq, nk, h, hk, d)
    q.fill_(1.0)
    k.fill_(float("-inf"))
    assert bool((run(q, k, v, work=work) == 0).all())
    v2 = v.clone()
    for value, key in ((float("inf"), 3), (float("nan"), nk // 2), (float("-inf"), nk - 1)):
        v2[0, key, hk - 1, 5] = value
        assert bool((run(q, k, v2, work=work) == 0).all()), (value, key)
    k[0, nk // 3] = 0.5
    v2 = v.clone()
    v2[0, 3, hk - 1, 5], v2[0, nk - 1, 0, 7] = float("inf"), float("-inf")
    want = v[:, nk // 3].repeat_interleave(h // hk, dim=1)[:, None].expand(1, nq, h, d).clone()
    assert bool((run(q, k, v, work=work) == want).all())
    want[:, :, h - h // hk:, 5], want[:, :, :h // hk, 7] = float("inf"), float("-inf")
    assert bool((run(q, k, v2, work=work) == want).all())
