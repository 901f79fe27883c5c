"""Encoders over batches of long sequences, whose activations pass 2 GiB and 32-bit offsets."""
import numpy as np
import pytest

from tests.common import infer, log, make_runtime
from tests.test_gpu_models_w4 import check_samples, encoder, padded

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d,group", [(64, 0), (128, 0), (128, 64)])
def test_activations_beyond_2_gib(d, group):
    # 81,920 rows of 16,384 bf16 values inside the feed-forward layers, 2.7 GB: the last sample lies behind the first 2 GiB, and the
    # third reaches across the middle, where the rows are shared out to two launches
    lens = [500, 1, 8300, 0, 300]
    log(f"5 x 16384 tokens, d {d}, groups of {group}")
    m = encoder(16384, 64, 2, group, layers=1, d=d, ffn=16384)
    ids = padded(5, 16384, lens)
    rt, (mid,) = make_runtime([m], batch_max=5)
    got = infer(rt, mid, m, ids)
    log("  computed")
    assert rt.resident(mid)
    check_samples(got, m, ids)
    again = infer(rt, mid, m, ids)
    rt.close()
    assert np.array_equal(got, again)
