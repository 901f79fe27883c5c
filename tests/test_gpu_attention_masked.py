"""tpo_attention against softmax attention in 64 bits: lengths, order, windows, sinks, shared heads, layouts."""
import math

import numpy as np
import pytest

from tests.common import log
from tests.ops_common import attention, seen

pytestmark = pytest.mark.gpu


def scratch():
    import paper_2306_03622_amd as tp
    import torch
    return torch.empty(tp.TPO_WORK_BYTES, dtype=torch.uint8, device="cuda:0").fill_(255)


def make(seed, b, qn, kn, h, hk, d, std=1.5):
    import torch
    g = torch.Generator(device="cuda:0")
    g.manual_seed(seed)
    r = lambda *s, std=1.0: (torch.randn(*s, generator=g, device="cuda:0") * std).to(torch.bfloat16)   # noqa: E731
    return r(b, qn, h, d, std=std), r(b, kn, hk, d), r(b, kn, hk, d)


def lens_tensor(v):
    import torch
    return None if v is None else torch.tensor(v, dtype=torch.int32, device="cuda:0")


def run(q, k, v, q_lens=None, kv_lens=None, work=True, stream=None, fill=5.0, **kw):
    import paper_2306_03622_amd as tp
    import torch
    out = torch.full(q.shape, fill, dtype=torch.bfloat16, device="cuda:0")
    torch.cuda.synchronize()
    tp.tpo_attention(q, k, v, out, q_lens=lens_tensor(q_lens), kv_lens=lens_tensor(kv_lens), work=scratch() if work else None,
                     stream=stream, **kw)
    torch.cuda.synchronize()
    return out


def check(q, k, v, out, q_lens=None, kv_lens=None, causal=False, window=(-1, -1), sinks=0, scale=0.0, fill=5.0, every=1):
    b, nq, h, d = q.shape
    nk, hk = k.shape[1], k.shape[2]
    Q, K, V, O = (t.double().cpu().numpy() for t in (q, k, v, out))
    worst = 0.0
    for i in range(b):
        qn = nq if q_lens is None else min(max(q_lens[i], 0), nq)
        kn = nk if kv_lens is None else min(max(kv_lens[i], 0), nk)
        assert (O[i, qn:] == fill).all(), "rows behind the last query were written"
        m = seen(qn, kn, causal, *window, sinks)
        for j in range(0, h, every):
            jk = j // (h // hk)
            want, tol = attention(Q[i, :qn, j], K[i, :kn, jk], V[i, :kn, jk], m, scale or 1 / math.sqrt(d))
            off = np.abs(O[i, :qn, j] - want)
            assert np.isfinite(O[i, :qn, j]).all()
            assert (off <= tol).all(), (i, j, float((off - tol).max()), np.unravel_index((off - tol).argmax(), off.shape))
            worst = max(worst, float((off / np.maximum(tol, 1e-30)).max(initial=0)))
    log(f"  worst share of the tolerance {worst:.2f}")


# (sequences, query heads, key/value heads, dim, queries, keys, options): single tokens over short and long caches, chunks, whole
# sequences; windows and sinks that end inside tiles; lengths of zero and one; more queries than tokens
CASES = [
    (1, 1, 1, 64, 1, 1, {}),
    (2, 2, 2, 128, 1, 33, {"causal": True}),
    (3, 8, 2, 128, 1, 700, {"causal": True, "kv_lens": [700, 1, 0], "q_lens": [1, 1, 1]}),
    (2, 32, 8, 128, 1, 2500, {"causal": True, "window": (300, 0), "sinks": 4, "kv_lens": [2500, 311]}),
    (1, 8, 1, 64, 1, 9000, {"causal": True}),
    (1, 4, 4, 128, 1, 5000, {"causal": True, "window": (1, 0), "sinks": 1}),
    (2, 6, 2, 64, 5, 400, {"causal": True, "kv_lens": [400, 3], "q_lens": [5, 5]}),
    (1, 16, 2, 128, 4, 3001, {"causal": True, "window": (1000, 0), "sinks": 70}),
    (5, 12, 12, 64, 96, 96, {"q_lens": [96, 80, 1, 0, 47], "kv_lens": [96, 80, 1, 0, 47]}),
    (2, 3, 3, 64, 32, 32, {}),
    (1, 2, 2, 128, 257, 257, {"causal": True}),
    (2, 4, 2, 64, 300, 300, {"window": (17, 5), "q_lens": [300, 129], "kv_lens": [300, 129]}),
    (1, 2, 1, 64, 1000, 1000, {"window": (64, 64), "sinks": 1}),
    (1, 2, 2, 128, 500, 500, {"window": (0, 0)}),
    (1, 2, 2, 64, 500, 500, {"window": (0, 0), "sinks": 3}),
    (1, 3, 1, 128, 333, 1500, {"causal": True, "window": (200, 0), "sinks": 130}),
    (2, 8, 4, 128, 150, 900, {"causal": True, "kv_lens": [900, 200], "q_lens": [150, 37]}),
    (1, 2, 2, 64, 200, 120, {"causal": True}),
    (1, 2, 2, 64, 200, 120, {"window": (30, 10), "sinks": 2}),
    (1, 2, 2, 64, 130, 400, {"window": (-1, 7)}),
    (1, 2, 2, 64, 130, 400, {"window": (9, -1), "sinks": 20}),
    (1, 4, 4, 128, 64, 64, {"sinks": 500, "window": (2, 2)}),
    (1, 2, 2, 64, 40, 40, {"causal": True, "scale": 0.5}),
    (2, 5, 1, 64, 77, 77, {"causal": True, "q_lens": [-3, 99], "kv_lens": [77, 1000]}),
    (1, 7, 7, 128, 33, 0, {}),
    (1, 24, 8, 64, 11, 260, {"causal": True}),
]


@pytest.mark.parametrize("i", range(len(CASES)))
def test_results(i):
    b, h, hk, d, nq, nk, kw = CASES[i]
    log(f"{b} x {nq} over {nk}, {h} / {hk} heads of {d}: {kw}")
    q, k, v = make(100 + i, b, nq, nk, h, hk, d)
    opts = dict(kw)
    for work in (True, False):
        out = run(q, k, v, work=work, **kw)
        check(q, k, v, out, **opts)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("nq,nk,causal,window,sinks", [
    (1, 1, True, (-1, -1), 0), (1, 4095, True, (-1, -1), 0), (1, 4095, True, (513, 0), 6), (3, 1029, True, (40, 0), 40), (64, 64, False, (3, 9), 0),
    (129, 129, True, (-1, -1), 0), (255, 700, True, (100, 0), 3), (400, 400, False, (31, 32), 65), (130, 2000, True, (1000, 0), 700)])
def test_exactly_the_seen_keys_count(d, nq, nk, causal, window, sinks):
    # queries of zeros weigh every seen key 1, exactly; a key's value is 1 in one column and 0 elsewhere, so a column holds
    # how many seen keys have it, over all of them: a count below 128 that the result's rounding (2^-8 of it) leaves
    # readable. Two sets of columns, by the key's place in a block of d and by its block of 16, tell which keys they are.
    import torch
    h, hk = 4, 2
    q = torch.zeros(1, nq, h, d, dtype=torch.bfloat16, device="cuda:0")
    _, k, _ = make(7, 1, 1, nk, h, hk, d)
    m = seen(nq, nk, causal, *window, sinks)
    j = np.arange(nk)
    for col in (j % d, j // 16 % d):
        one = np.zeros((nk, d))
        one[j, col] = 1
        v = torch.tensor(one, device="cuda:0").to(torch.bfloat16).view(1, nk, 1, d).expand(1, nk, hk, d).contiguous()
        for work in (True, False):
            out = run(q, k, v, work=work, causal=causal, window=window, sinks=sinks)[0].double().cpu().numpy()
            want, all_ = m @ one, m.sum(axis=1)
            assert want.max() < 128
            for head in range(h):
                assert np.array_equal(np.rint(out[:, head] * all_[:, None]), want), head


# shapes for each way of cutting the rows and keys, most of which small ones do not take: rows in 32s, 64s, 128s and 256s, waves
# one, two and four deep, the keys split or not (the comment in attn_masked.hip names the limits)
LARGE = [(64, 9, 9, 70, 2000, {"causal": True}), (64, 530, 530, 130, 1100, {"causal": True, "window": (1040, 0), "sinks": 3}), (64, 210, 210, 70, 90, {}), (64, 530, 530, 130, 150, {"window": (40, 3), "sinks": 2}),
         (128, 100, 100, 70, 300, {"causal": True}), (128, 60, 60, 150, 300, {"causal": True}), (128, 8, 4, 120, 3000, {"causal": True, "window": (2000, 0), "sinks": 5}),
         (128, 300, 300, 100, 200, {"window": (64, 64)}), (128, 530, 530, 100, 260, {"causal": True, "window": (100, 0), "sinks": 1}),
         (128, 530, 530, 70, 2300, {"causal": True}), (128, 1060, 530, 75, 2100, {"window": (2050, 30)}),
         (64, 16, 8, 3, 33000, {"causal": True}), (128, 32, 8, 2, 17000, {"causal": True, "window": (16500, 0), "sinks": 9})]


@pytest.mark.parametrize("i", range(len(LARGE)))
def test_large(i):
    d, h, hk, nq, nk, kw = LARGE[i]
    log(f"{nq} over {nk}, {h} / {hk} heads of {d}: {kw}")
    q, k, v = make(500 + i, 1, nq, nk, h, hk, d)
    out = run(q, k, v, **kw)
    check(q, k, v, out, every=max(1, h // 7), **kw)
    # hidden infinities and NaN change nothing; a seen one shows in its column of the rows that see it
    m = seen(nq, nk, kw.get("causal", False), *kw.get("window", (-1, -1)), kw.get("sinks", 0))
    k2, v2 = k.clone(), v.clone()
    for j in np.flatnonzero(~m.any(axis=0))[:40]:
        k2[:, int(j)], v2[:, int(j)] = float("nan"), float("inf")
    j = int(np.flatnonzero(m.any(axis=0) & ~m.all(axis=0))[-1]) if (m.any(axis=0) & ~m.all(axis=0)).any() else nk - 1
    v2[0, j, hk // 2, 11] = float("-inf")
    got, want = run(q, k2, v2, **kw), out.clone()
    for head in range(hk // 2 * (h // hk), (hk // 2 + 1) * (h // hk)):
        for i in np.flatnonzero(m[:, j]):
            want[0, int(i), head, 11] = float("-inf")
    assert bool((got == want).all())


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("nq,nk", [(1, 2000), (4, 300), (200, 200), (150, 900)])
def test_hidden_keys_may_hold_anything(d, nq, nk):
    # infinities and NaN in keys and values that no query sees, in and behind the sequence
    kn = nk - 3
    qn = min(nq, kn)
    q, k, v = make(31 + nq, 2, nq, nk, 4, 2, d)
    kw = {"causal": True, "window": (40, 0), "sinks": 2, "q_lens": [qn, qn], "kv_lens": [kn, kn]}
    clean = run(q, k, v, **kw)
    lo = kn - qn - 40                       # the first key that the window reaches
    for value in (float("nan"), float("inf"), float("-inf")):
        k2, v2 = k.clone(), v.clone()
        for t in (k2, v2):
            t[:, kn:] = value
            if lo > 2:
                t[:, 2:lo] = value
        got = run(q, k2, v2, **kw)
        assert bool((got == clean).all()), value


@pytest.mark.parametrize("nq,nk", [(1, 500), (180, 180)])
def test_odd_values_reach_only_who_sees_them(nq, nk):
    # one key whose value holds an infinity (or NaN): the rows that see it, in that column, and no others
    import torch
    q, k, v = make(77, 1, nq, nk, 2, 1, 64)
    kw = {"causal": True, "window": (30, 0), "sinks": 1}
    clean = run(q, k, v, **kw)
    m = seen(nq, nk, True, 30, 0, 1)
    for key in (0, nk - 31, nk - 1, nk // 2):
        for value in (float("inf"), float("-inf"), float("nan")):
            v2 = v.clone()
            v2[0, key, 0, 9] = value
            got = run(q, k, v2, **kw)[0]
            sees = torch.tensor(m[:, key], device="cuda:0")
            want = clean[0].clone()
            want[sees, :, 9] = value
            assert bool(torch.equal(torch.nan_to_num(got, 1e4, 2e4, -2e4), torch.nan_to_num(want, 1e4, 2e4, -2e4))), (key, value)
    both = v.clone()
    both[0, nk - 1, 0, 3], both[0, nk - 2, 0, 3] = float("inf"), float("-inf")
    assert bool(run(q, k, both, **kw)[0, -1, :, 3].isnan().all())


def test_layouts():
    # slices of one projection, a cache with room behind, heads before tokens, a broadcast key/value head
    import torch
    g = torch.Generator(device="cuda:0")
    g.manual_seed(1)
    b, s, h, d = 2, 150, 3, 64
    qkv = torch.randn(b, s, 3 * h, d, generator=g, device="cuda:0").to(torch.bfloat16)
    q, k, v = qkv[:, :, :h], qkv[:, :, h:2 * h], qkv[:, :, 2 * h:]
    for kw in ({}, {"causal": True, "window": (20, 0)}):
        check(q, k, v, run(q, k, v, **kw), **kw)
        t = lambda x: x.transpose(1, 2).contiguous().transpose(1, 2)   # noqa: E731
        assert bool((run(t(q), t(k), t(v), **kw) == run(q, k, v, **kw)).all())
    room = torch.full((b, s + 40, h, d), float("nan"), dtype=torch.bfloat16, device="cuda:0")
    room[:, :s] = k
    assert bool((run(q, room[:, :s], v, causal=True) == run(q, k, v, causal=True)).all())
    kb, vb = k[:, :, :1].expand(b, s, h, d), v[:1, :, :1].expand(b, s, h, d)
    check(q, kb, vb, run(q, kb, vb))
    # an output with gaps, which stay
    import paper_2306_03622_amd as tp
    wide = torch.full((b, s, h, d + 8), 3.0, dtype=torch.bfloat16, device="cuda:0")
    tp.tpo_attention(q, k, v, wide[..., :d], causal=True)
    assert bool((wide[..., d:] == 3).all()) and bool((wide[..., :d] == run(q, k, v, causal=True)).all())


def test_offsets_beyond_32_bits():
    # tokens so far apart that the last lies 5 GiB behind the first
    import torch
    nk, d, step = 320, 64, 1 << 23
    k = torch.zeros(nk * step + d, dtype=torch.bfloat16, device="cuda:0").as_strided((1, nk, 1, d), (0, step, 0, 1))
    q, k0, v = make(3, 1, 40, nk, 1, 1, d)
    k.copy_(k0)
    assert bool((run(q, k, v, causal=True) == run(q, k0, v, causal=True)).all())
    assert bool((run(q, v, k, causal=True) == run(q, v, k0, causal=True)).all())


def test_streams_and_graphs():
    import paper_2306_03622_amd as tp
    import torch
    for nq, nk, kw in ((1, 3000, {"causal": True}), (90, 500, {"causal": True, "window": (64, 0), "sinks": 2})):
        sets = [make(200 + i, 2, nq, nk, 8, 2, 128) for i in range(3)]
        lens = [[nk, nk // 2 + i * 7] for i in range(3)]
        want = [run(*s, kv_lens=l, **kw) for s, l in zip(sets, lens)]
        side = torch.cuda.Stream(device="cuda:0")
        assert bool((run(*sets[0], kv_lens=lens[0], stream=side, **kw) == want[0]).all())
        q, k, v = (t.clone() for t in sets[0])
        kl, work, out = lens_tensor(lens[0]), scratch(), torch.empty_like(q)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            tp.tpo_attention(q, k, v, out, kv_lens=kl, work=work, **kw)
        for i in (1, 2, 0, 1):
            for dst, src in zip((q, k, v), sets[i]):
                dst.copy_(src)
            kl.copy_(lens_tensor(lens[i]))
            out.fill_(-9)
            tp.tpo_attention(*sets[2], torch.empty_like(q), work=work, **kw)      # an eager call between the replays
            g.replay()
            torch.cuda.synchronize()
            assert bool((out == want[i]).all())
