"""Values of the operators' arguments that leave the range of the kernels' arithmetic (no GPU: refused before a launch)."""
import numpy as np
import pytest

import paper_2306_03622_amd as tp
from tests.test_ops_host import _status, attention_args


@pytest.mark.parametrize("scale,ok", [(np.finfo(np.float32).max, False), (float(np.nextafter(np.float32(2.0 ** 127), np.float32(np.inf))), False),
                                      (2.0 ** 127, True), (1e-45, True), (-1e-45, False)])
def test_scales(scale, ok):
    # times log2(e), as the kernels use it, a scale stays finite: 2^127 * 1.4427 < 2^128
    with np.errstate(over="ignore"):
        assert np.isfinite(np.float32(scale) * np.float32(1.44269504)) or not ok
    st, msg = _status("tpo_attention", attention_args(scale=scale, batch=0))      # a call of nothing: the checks alone
    assert (st == tp.TP_OK) == ok and (ok or "scale" in msg)
