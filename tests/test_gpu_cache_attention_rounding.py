"""tps_cache_attention's own roundings: every kernel within what two bf16 parts of an exponential leave, and infinite values."""
import math

import numpy as np
import pytest

from tests.common import log
from tests.serve_common import seen
from tests.test_gpu_cache_attention import Setup
from tests.test_gpu_serve_variants import ATTENTION, PAIRS

pytestmark = pytest.mark.gpu


def reference(q, k, v, m, scale):
    """One head of one sequence -> (out, tolerance), elementwise. An exponential's first bf16 part leaves less than 2^-7 of it, the second
    2^-8 of that: 2^-15. The result is rounded once (2^-8 of it). Scores, exponentials and sums are fp32: a dot product of d terms is off by
    at most d 2^-23 of sum |q k|, which moves an exponential by as much of itself (once in the sum that divides, once in the one that is
    divided); the hardware exponential, the running rescaling and the sums add less than 1e-5."""
    s = np.where(m, (q @ k.T) * scale, -np.inf)
    e = np.exp(s - s.max(axis=1, keepdims=True))
    w = e / e.sum(axis=1, keepdims=True)
    out, size = w @ v, w @ np.abs(v)
    spread = float((np.where(m, np.abs(q) @ np.abs(k).T, 0) * scale).max())
    return out, 2.0 ** -8 * np.abs(out) + (2.0 ** -15 + 1e-5 + 2 * q.shape[1] * 2.0 ** -23 * spread) * (1 + 2.0 ** -8) * size


@pytest.mark.parametrize("dim,e4m3,i", [(d, e, i) for (d, e), more in PAIRS.items() for i in range(len(ATTENTION) + len(more))])
def test_exponentials_keep_sixteen_bits(dim, e4m3, i):
    kernel, nq, h, hk, page, lens, kw = (ATTENTION + PAIRS[dim, e4m3])[i]
    log(f"{kernel} {nq} over {lens}, {h} / {hk} heads of {dim}")
    # scores of about 0.25 (no exponential is much larger than the others), values that cancel each other
    s = Setup(900 + i, len(lens), nq, h, hk, dim, page, lens, e4m3, std=0.25)
    out = s.run(**kw).double().cpu().numpy()
    Q, pool, worst = s.q.double().cpu().numpy(), s.pool(), 0.0
    for b, kn in enumerate(lens):
        first = max(0, nq - kn)                     # (rows in front of token 0 see nothing)
        k, v, _ = pool.sequence(b, kn)
        m = seen(nq, kn, kw.get("window", -1), kw.get("sinks", 0))[first:]
        for j in range(0, h, max(1, h // 8)):
            want, tol = reference(Q[b, first:, j], k[:, j // (h // hk)], v[:, j // (h // hk)], m, 1 / math.sqrt(dim))
            off = np.abs(out[b, first:, j] - want)
            assert (off <= tol).all(), (b, j, float((off / tol).max()))
            worst = max(worst, float((off / tol).max()))
    log(f"  worst share of the tolerance {worst:.2f}")


@pytest.mark.parametrize("dim", [64, 128])
def test_an_infinite_value_is_that_infinity(dim):
    # of keys of any weight, exactly 1 among them, in tiles that hold hidden keys and in whole ones; no other column shows it
    kn, page = 200, 16
    for at, sign in ((0, 1), (37, -1), (64, 1), (199, -1)):
        for std in (0.0, 0.5, 4.0):
            s = Setup(60, 1, 2, 4, 2, dim, page, [kn], False, std=std)
            clean = s.run()
            s.v[s.table[0][at // page], at % page, 1, 9] = sign * math.inf
            out = s.run()
            want = clean.clone()
            want[0, :, 2:, 9] = sign * math.inf
            if at == kn - 1:
                want[0, 0] = clean[0, 0]            # (the first of the two does not see the last token)
            assert bool((out == want).all()), (at, std)


def test_opposite_infinities_are_nan():
    import torch
    s = Setup(61, 1, 1, 2, 1, 64, 16, [100], False)
    s.v[s.table[0][0], 3, 0, 5], s.v[s.table[0][2], 3, 0, 5] = math.inf, -math.inf
    out = s.run()
    assert bool(torch.isnan(out[..., 5]).all()) and int(torch.isnan(out).sum()) == 2
