"""Every kernel of tpo_attention, with its keys split over workgroups and not, on ragged batches: sequences without queries, without
keys, with fewer keys than queries and with lengths out of range. test_attn_plan.py checks that the shapes take the kernels they name."""
import numpy as np
import pytest

from tests.common import log
from tests.ops_common import seen
from tests.test_gpu_attention_masked import check, lens_tensor, make, run, scratch

pytestmark = pytest.mark.gpu

# kernel, split; sequences, query heads, key/value heads, dim, queries, keys, options
SHAPES = [
    ("ATTN64_R32", False, 3, 4, 2, 64, 5, 1100, {"causal": True, "window": (120, 0), "sinks": 3}),
    ("ATTN64_R32", True, 3, 4, 2, 64, 5, 1100, {"causal": True}),
    ("ATTN64_R64", False, 3, 90, 90, 64, 5, 1100, {"causal": True, "window": (1000, 0), "sinks": 70}),
    ("ATTN64_R64", True, 3, 8, 2, 64, 20, 2500, {"causal": True}),
    ("ATTN64_R128", False, 3, 90, 90, 64, 200, 260, {"window": (40, 70), "sinks": 2}),
    ("ATTN64_R128_LONG", False, 3, 180, 180, 64, 130, 1500, {"causal": True}),
    ("ATTN128_R32", False, 3, 4, 2, 128, 5, 1100, {"causal": True, "window": (120, 0), "sinks": 3}),
    ("ATTN128_R32", True, 3, 4, 2, 128, 5, 1100, {"causal": True}),
    ("ATTN128_R64", False, 3, 90, 90, 128, 5, 1100, {"causal": True}),
    ("ATTN128_R64", True, 3, 24, 6, 128, 3, 9000, {"causal": True}),
    ("ATTN128_R128_DEEP", False, 3, 32, 8, 128, 200, 260, {"causal": True, "window": (90, 0), "sinks": 1}),
    ("ATTN128_R128_DEEP", True, 3, 4, 2, 128, 130, 1500, {"causal": True}),
    ("ATTN128_R128", False, 3, 96, 24, 128, 100, 300, {"causal": True}),
    ("ATTN128_R128", False, 3, 96, 24, 128, 131, 700, {"window": (300, 9), "sinks": 5}),
    ("ATTN128_R256", False, 3, 171, 171, 128, 70, 2100, {"causal": True}),
]


def lengths(b, nq, nk, turn):
    """Queries and keys of each sequence; the last has fewer keys than queries."""
    q = [[nq, nq // 2 + 1, nq], [0, nq, nq], [-3, nq + 50, 1]][turn]
    k = [[nk, nk // 2, max(1, nq // 2)], [nk, 0, max(1, nq // 3)], [nk, nk + 1000, max(1, nk - 40)]][turn]
    return {"q_lens": q[:b], "kv_lens": k[:b]}


@pytest.mark.parametrize("i", range(len(SHAPES)))
def test_ragged_batches(i):
    name, split, b, h, hk, d, nq, nk, kw = SHAPES[i]
    q, k, v = make(900 + i, b, nq, nk, h, hk, d)
    for turn in range(3):
        lens = lengths(b, nq, nk, turn)
        log(f"{name}, split {split}: {lens}")
        check(q, k, v, run(q, k, v, work=split, **lens, **kw), every=max(1, h // 6), **lens, **kw)


@pytest.mark.parametrize("i", range(len(SHAPES)))
def test_hidden_values_and_seen_ones(i):
    name, split, b, h, hk, d, nq, nk, kw = SHAPES[i]
    log(f"{name}, split {split}")
    q, k, v = make(930 + i, b, nq, nk, h, hk, d)
    lens = lengths(b, nq, nk, 0)
    want = run(q, k, v, work=split, **lens, **kw)
    k2, v2 = k.clone(), v.clone()
    masks = []
    for s, (qn, kn) in enumerate(zip(lens["q_lens"], lens["kv_lens"])):
        m = seen(qn, kn, kw.get("causal", False), *kw.get("window", (-1, -1)), kw.get("sinks", 0))
        masks.append(m)
        k2[s, kn:], v2[s, kn:] = float("inf"), float("nan")
        hidden = np.flatnonzero(~m.any(axis=0))
        if len(hidden):
            at = lens_tensor(hidden.tolist()).long()
            k2[s, at], v2[s, at] = float("nan"), float("-inf")
    assert bool((run(q, k2, v2, work=split, **lens, **kw) == want).all())
    # one seen infinity per sequence: its column, in the rows and heads that see it
    share = h // hk
    for s, m in enumerate(masks):
        key = int(np.flatnonzero(m.any(axis=0))[-1])
        v2[s, key, hk - 1, 11 + s] = float("inf")
        rows = lens_tensor(np.flatnonzero(m[:, key]).tolist()).long()
        want[s, rows, (hk - 1) * share:, 11 + s] = float("inf")
    assert bool((run(q, k2, v2, work=split, **lens, **kw) == want).all())


@pytest.mark.parametrize("i", range(len(SHAPES)))
def test_replays_with_other_lengths(i):
    import paper_2306_03622_amd as tp
    import torch
    name, split, b, h, hk, d, nq, nk, kw = SHAPES[i]
    log(f"{name}, split {split}")
    q, k, v = make(960 + i, b, nq, nk, h, hk, d)
    want = [run(q, k, v, work=split, fill=-9.0, **lengths(b, nq, nk, t), **kw) for t in range(3)]
    first = lengths(b, nq, nk, 0)
    ql, kl = lens_tensor(first["q_lens"]), lens_tensor(first["kv_lens"])
    work, out = scratch() if split else None, torch.empty_like(q)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        tp.tpo_attention(q, k, v, out, q_lens=ql, kv_lens=kl, work=work, **kw)
    for t in (1, 2, 0, 1):
        lens = lengths(b, nq, nk, t)
        ql.copy_(lens_tensor(lens["q_lens"]))
        kl.copy_(lens_tensor(lens["kv_lens"]))
        out.fill_(-9)
        tp.tpo_attention(q, k, v, torch.empty_like(q), work=work, **kw)           # an eager call between the replays
        g.replay()
        torch.cuda.synchronize()
        assert bool((out == want[t]).all())
