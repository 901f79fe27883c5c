"""tps_cache_attention against softmax attention in 64 bits: lengths, pages, windows, sinks, drafted tokens, layouts, 8-bit caches."""
import math

import numpy as np
import pytest

from tests.common import log
from tests.serve_common import Pool, cache_attention, e4m3_values, seen
from tests.test_gpu_cache_rows import dev, table_of

pytestmark = pytest.mark.gpu


def scratch():
    import paper_2306_03622_amd as tp
    import torch
    return torch.empty(tp.TPO_WORK_BYTES, dtype=torch.uint8, device="cuda:0").fill_(255)


class Setup:
    """Random pages; a table that names each page once; queries."""

    def __init__(self, seed, batch, qn, heads, kv_heads, dim, page, kv_lens, e4m3, std=1.5, order="tokens", spare=2):
        import paper_2306_03622_amd as tp
        import torch
        rng = np.random.default_rng(seed)
        g = torch.Generator(device="cuda:0")
        g.manual_seed(seed)
        columns = max(1, max((n + page - 1) // page for n in kv_lens))
        pages = batch * columns + spare
        self.table = table_of(rng, batch, columns, pages)
        self.kv_lens, self.page, self.e4m3 = kv_lens, page, e4m3
        shape = (pages, kv_heads, page, dim) if order == "heads" else (pages, page, kv_heads, dim)
        pool = [torch.randn(*shape, generator=g, device="cuda:0") for _ in "kv"]
        self.exps = None
        if e4m3:
            pool = [(t * 100).clamp(-448, 448).to(torch.float8_e4m3fn) for t in pool]
            self.exps = torch.randint(117, 122, (pages, 2, kv_heads, page), generator=g, device="cuda:0").to(torch.uint8)
        else:
            pool = [t.to(torch.bfloat16) for t in pool]
        self.k, self.v = (t.transpose(1, 2) if order == "heads" else t for t in pool)
        self.cache = tp.PagedCache(self.k, self.v, self.exps)
        self.q = (torch.randn(batch, qn, heads, dim, generator=g, device="cuda:0") * std).to(torch.bfloat16)

    def pool(self):
        import torch
        out = []
        for n, t in enumerate((self.k, self.v)):
            if self.e4m3:
                x = e4m3_values()[t.contiguous().view(torch.uint8).cpu().numpy()]
                x = x * 2.0 ** (self.exps[:, n].cpu().numpy().astype(np.float64) - 127).transpose(0, 2, 1)[..., None]
            else:
                x = t.double().cpu().numpy()
            out.append(x)
        return Pool(*out, self.table, self.page)

    def run(self, q_lens=None, work=True, fill=5.0, table=None, kv_len=None, stream=None, **kw):
        import paper_2306_03622_amd as tp
        import torch
        out = torch.full(self.q.shape, fill, dtype=torch.bfloat16, device="cuda:0")
        i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda:0")       # noqa: E731
        args = (dev(self.table if table is None else table), i32(self.kv_lens))
        w = scratch() if work else None
        ql = None if q_lens is None else i32(q_lens)
        torch.cuda.synchronize()
        tp.tps_cache_attention(self.cache, *args, self.q, out, q_lens=ql, kv_len=kv_len, work=w, stream=stream, **kw)
        torch.cuda.synchronize()
        return out

    def check(self, out, q_lens=None, window=-1, sinks=0, scale=0.0, fill=5.0, kv_len=None, every=1, pool=None, skip=None):
        """pool: values of another time; skip: places of the result that are not compared."""
        b, nq, h, d = self.q.shape
        hk = self.cache.kv_heads
        Q, O, pool = self.q.double().cpu().numpy(), out.double().cpu().numpy(), pool or self.pool()
        if skip is not None:
            O = np.where(skip.cpu().numpy(), np.nan, O)
        worst = 0.0
        for i in range(b):
            qn = nq if q_lens is None else min(max(q_lens[i], 0), nq)
            kn = max(self.kv_lens[i], 0) if kv_len is None else min(max(self.kv_lens[i], 0), kv_len)
            kn = min(kn, self.table.shape[1] * self.page)
            assert (O[i, qn:] == fill).all(), "rows behind the last query were written"
            k, v, there = pool.sequence(i, kn)
            m = seen(qn, kn, window, sinks) & there[None]
            for j in range(0, h, every):
                want, tol = cache_attention(Q[i, :qn, j], k[:, j // (h // hk)], v[:, j // (h // hk)], m, scale or 1 / math.sqrt(d))
                off = np.abs(O[i, :qn, j] - want)
                if skip is not None:
                    off[skip[i, :qn, j].cpu().numpy()] = 0
                assert np.isfinite(off).all(), (i, j)
                assert (off <= tol).all(), (i, j, float((off - tol).max()), np.unravel_index((off - tol).argmax(), off.shape))
                worst = max(worst, float((off / np.maximum(tol, 1e-30)).max(initial=0)))
        log(f"  worst share of the tolerance {worst:.2f}")


# (new tokens, heads, key/value heads, dim, page, lengths, options)
CASES = [
    (1, 1, 1, 64, 16, [1], {}),
    (1, 2, 2, 128, 16, [33, 1], {}),
    (1, 8, 2, 128, 32, [700, 1, 0], {}),
    (1, 32, 8, 128, 16, [2500, 311], {"window": 300, "sinks": 4}),
    (1, 8, 1, 64, 64, [9000], {}),
    (1, 12, 4, 128, 256, [5000], {"window": 1, "sinks": 1}),
    (5, 6, 2, 64, 16, [400, 3], {"q_lens": [5, 5]}),
    (4, 16, 2, 128, 128, [3001], {"window": 1000, "sinks": 70}),
    (8, 8, 1, 128, 32, [1000, 37, 8], {"q_lens": [8, 0, 3]}),
    (7, 24, 8, 64, 16, [260], {}),
    (1, 7, 7, 128, 16, [0], {}),
    (2, 3, 3, 64, 16, [513, 512], {"window": 0}),
    (2, 3, 1, 64, 16, [513, 31], {"window": 0, "sinks": 3}),
    (16, 4, 1, 128, 32, [600], {"scale": 0.5}),
    (100, 4, 2, 128, 16, [100, 40], {"q_lens": [100, 40]}),
    (130, 4, 2, 64, 64, [1030], {"window": 200, "sinks": 33}),
    (3, 5, 1, 64, 4096, [77, 5000], {"q_lens": [-3, 99]}),
    (1, 40, 1, 128, 16, [90, 4], {}),
    (1, 64, 2, 64, 16, [90], {}),
    (4, 2, 2, 64, 16, [200], {"kv_len": 100}),
]


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("i", range(len(CASES)))
def test_results(i, e4m3):
    nq, h, hk, d, page, kv_lens, kw = CASES[i]
    log(f"{nq} over {kv_lens}, {h} / {hk} heads of {d}, pages of {page}: {kw}")
    s = Setup(100 + i, len(kv_lens), nq, h, hk, d, page, kv_lens, e4m3, order="heads" if i % 3 == 1 else "tokens")
    for work in (True, False):
        s.check(s.run(work=work, **kw), **kw)


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("nq,nk,window,sinks,page", [(1, 1, -1, 0, 16), (1, 4095, -1, 0, 16), (1, 4095, 513, 6, 32), (3, 1029, 40, 40, 16),
                                                     (8, 700, 100, 3, 64), (20, 2000, 1000, 700, 16), (2, 65, 0, 1, 32)])
def test_exactly_the_seen_keys_count(d, nq, nk, window, sinks, page, e4m3):
    # queries of zeros weigh every seen key 1, exactly; a key's value is 1 in one column and 0 elsewhere, so a column times the count
    # of seen keys is how many of them have it, a whole number below 128, which the result's rounding (2^-8 of it) leaves readable
    import torch
    h, hk = 4, 2
    s = Setup(7, 1, nq, h, hk, d, page, [nk], e4m3)
    s.q.zero_()
    m = seen(nq, nk, window, sinks)
    j = np.arange(nk)
    place = s.table[0][j // page], j % page
    for col in (j % d, j // 16 % d):
        one = np.zeros((s.v.shape[0], page, hk, d), dtype=np.float32)
        one[place[0], place[1], :, col] = 1
        s.v.copy_(torch.from_numpy(one).to(s.v.dtype))
        if e4m3:
            s.exps[:, 1] = 127
        out = s.run(window=window, sinks=sinks).double().cpu().numpy()
        hot = np.eye(d)[col]
        want = m @ hot                                  # [nq][d]
        n = m.sum(axis=1)
        assert want.max() < 128
        got = out[0] * n[:, None, None]
        assert (np.rint(got) == want[:, None, :]).all()
        assert (np.abs(got - want[:, None]) <= 2.0 ** -8 * want[:, None] * 1.01).all()


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("bad", ["nan", "inf"])
def test_hidden_places_may_hold_anything(e4m3, bad):
    # places behind the last token, left of the window and right of a drafted token, spare pages: all of them not finite
    import torch
    nq, kn, window, sinks, page, d = 6, 300, 50, 5, 32, 64
    s = Setup(31, 2, nq, 4, 2, d, page, [kn, 200], e4m3)
    s.check(s.run(window=window, sinks=sinks), window=window, sinks=sinks)
    clean = s.pool()
    raw = lambda t: t.view(torch.uint8) if e4m3 else t                           # noqa: E731
    poison = 0x7F if e4m3 else float(bad)
    keep = np.zeros(s.k.shape[:2], dtype=bool)
    for b, n in enumerate(s.kv_lens):
        used = np.nonzero(seen(nq, n, window, sinks).any(axis=0))[0]
        keep[s.table[b][used // page], used % page] = True
    gone = torch.from_numpy(~keep).to("cuda:0")
    for t in (s.k, s.v):
        raw(t)[gone] = poison
    if e4m3:
        s.exps.copy_(torch.where(gone[:, None, None, :], 255, s.exps.int()).to(torch.uint8))
    s.check(s.run(window=window, sinks=sinks), window=window, sinks=sinks, pool=clean)
    # the newest token's value is not finite: it shows to the last query of its sequence, in its column, and to no other
    last = s.table[0][(kn - 1) // page], (kn - 1) % page
    raw(s.v)[last[0], last[1], 1, 9] = poison
    out = s.run(window=window, sinks=sinks)
    odd = ~torch.isfinite(out)
    want = torch.zeros_like(odd)
    want[0, nq - 1, 2:, 9] = True
    assert bool((odd == want).all())
    s.check(out, window=window, sinks=sinks, pool=clean, skip=want)


@pytest.mark.parametrize("e4m3", [False, True])
def test_scores_that_are_not_finite(e4m3):
    import torch
    if e4m3:
        s = Setup(5, 1, 3, 2, 1, 64, 16, [100], True)
        s.k.view(torch.uint8)[s.table[0][0], 3] = 0x7F                            # a NaN key that all see
        assert bool(torch.isnan(s.run()).all())
        assert not bool(torch.isnan(s.run(window=50)).any())
        return
    s = Setup(5, 1, 3, 2, 1, 64, 16, [100], False)
    s.q.abs_()
    s.k[...] = -float("inf")
    s.v[s.table[0][0], 3, 0, 7] = float("inf")
    assert not bool(s.run().any())                                                # every score -infinity: zeros, whatever the values hold
    s.k[s.table[0][2], 5] = 1.0                                                   # one key that counts: token 37
    out = s.run(window=90)
    want = s.v[s.table[0][2], 5, 0].expand(3, 2, 64)
    assert bool((out[0] == want).all())


@pytest.mark.parametrize("e4m3", [False, True])
def test_pages_that_are_none(e4m3):
    # entries outside the pool hold no keys, wherever they stand; with none left a query gives zeros
    s = Setup(17, 3, 2, 8, 2, 128, 16, [500, 64, 16], e4m3)
    full = s.table.copy()
    s.table[0, 3], s.table[0, 10:14], s.table[0, 31] = -1, len(s.k), 2 ** 31 - 1
    s.table[1, :3] = -5
    s.table[2, :] = -1
    out = s.run()
    s.check(out)
    assert not bool(out[2].any())
    # pages that a window has left may be taken
    s.table = full
    want = s.run(window=100, sinks=2)
    taken = full.copy()
    for b, n in enumerate(s.kv_lens):
        taken[b, 1:max(1, (n - 2 - 100) // 16)] = -1
    assert bool((s.run(window=100, sinks=2, table=taken) == want).all())


def test_shared_pages():
    # sequences that share their first pages, and one that names a page twice
    s = Setup(19, 3, 1, 4, 2, 64, 16, [100, 90, 48], False)
    s.table[1, :4] = s.table[0, :4]
    s.table[2, 2] = s.table[2, 0]
    s.check(s.run())


def test_layouts():
    import paper_2306_03622_amd as tp
    import torch
    s = Setup(23, 3, 4, 6, 3, 64, 16, [70, 64, 5], False)
    want = s.run()
    g = s.q
    for q in (torch.cat((g, g), dim=3)[..., :64], g.transpose(1, 2).contiguous().transpose(1, 2), g[:, :1].expand(3, 4, 6, 64)):
        out = torch.full((3, 6, 4, 72), 5.0, dtype=torch.bfloat16, device="cuda:0").transpose(1, 2)[..., :64]
        table = torch.cat((dev(s.table), dev(s.table)), dim=1)[:, :s.table.shape[1]]
        tp.tps_cache_attention(s.cache, table, torch.tensor(s.kv_lens, dtype=torch.int32, device="cuda:0"), q, out, work=scratch())
        if q.stride(1) == 0:                          # one query for all tokens
            t = Setup(23, 3, 4, 6, 3, 64, 16, [70, 64, 5], False)
            t.q.copy_(q)
            want = t.run()
        assert bool((out == want).all())
    # a table of one column whose row stride is 0 for one sequence alone
    one = Setup(29, 1, 1, 2, 1, 64, 64, [60], False)
    one.check(one.run())


def test_long_cache_whose_offsets_pass_32_bits():
    # pages of a pool of 6 GiB: places beyond 2^32 bytes
    import paper_2306_03622_amd as tp
    import torch
    page, hk, d = 64, 8, 128
    pages = (6 << 30) // (page * hk * d * 2)
    k = torch.empty(pages, page, hk, d, dtype=torch.bfloat16, device="cuda:0")
    v = torch.empty_like(k)
    cache = tp.PagedCache(k, v)
    n = 5 * page - 3
    x = torch.randn(2, 1, n, hk, d, device="cuda:0").to(torch.bfloat16)
    table = torch.tensor([[pages - 1, 7, pages // 2, pages - 9, 3 * pages // 4]], dtype=torch.int32, device="cuda:0")
    lens = torch.tensor([n], dtype=torch.int32, device="cuda:0")
    tp.tps_cache_append(cache, table, lens, x[0], x[1])
    back = torch.zeros_like(x)
    tp.tps_cache_read(cache, table, lens, back[0], back[1])
    assert bool((back == x).all())
    q = torch.randn(1, 2, 16, d, device="cuda:0").to(torch.bfloat16)
    out = torch.zeros_like(q)
    tp.tps_cache_attention(cache, table, lens, q, out, work=scratch())
    Q, K, V, O = (t.double().cpu().numpy() for t in (q, x[0], x[1], out))
    for h in range(16):
        want, tol = cache_attention(Q[0, :, h], K[0, :, h // 2], V[0, :, h // 2], seen(2, n, -1, 0), d ** -0.5)
        assert (np.abs(O[0, :, h] - want) <= tol).all()


def test_streams_and_captured_graphs():
    import paper_2306_03622_amd as tp
    import torch
    setups = [Setup(41, 2, 1, 8, 2, 128, 16, [3000, 900], False), Setup(42, 2, 3, 8, 2, 64, 32, [2000, 1999], True)]
    calls, want = [], []
    for s in setups:
        out, work = torch.zeros_like(s.q), scratch()
        table, lens = dev(s.table), torch.tensor(s.kv_lens, dtype=torch.int32, device="cuda:0")
        calls.append((lambda s=s, out=out, work=work, table=table, lens=lens:
                      tp.tps_cache_attention(s.cache, table, lens, s.q, out, work=work), out))
        want.append(s.run())
        s.check(want[-1])
    streams = [torch.cuda.Stream(device="cuda:0") for _ in calls]
    torch.cuda.synchronize()
    for _ in range(20):
        for (call, _), stream in zip(calls, streams):
            with torch.cuda.stream(stream):
                call()
    torch.cuda.synchronize()
    assert all(bool((o == w).all()) for (_, o), w in zip(calls, want))
    graphs = []
    for call, _ in calls:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            call()
        graphs.append(g)
    for turn in range(4):
        for _, o in calls:
            o.fill_(-3)
        torch.cuda.synchronize()
        for g, stream in zip(graphs, streams):
            with torch.cuda.stream(stream):
                g.replay()
        torch.cuda.synchronize()
        assert all(bool((o == w).all()) for (_, o), w in zip(calls, want)), turn
