"""tps_lora against the adapters' products in 64 bits: mixed and grouped rows, ragged ranks, types, odd sizes, layouts."""
import numpy as np
import pytest

from tests.common import log
from tests.serve_common import lora

pytestmark = pytest.mark.gpu


def scratch():
    import paper_2306_03622_amd as tp
    import torch
    return torch.empty(tp.TPO_WORK_BYTES, dtype=torch.uint8, device="cuda:0").fill_(255)


class Setup:
    def __init__(self, seed, m, k, n, r, slots, f32, adapter, ranks=None, scales=True, base=True):
        import torch
        g = torch.Generator(device="cuda:0")
        g.manual_seed(seed)
        bf = lambda *s, std=1.0: (torch.randn(*s, generator=g, device="cuda:0") * std).to(torch.bfloat16)      # noqa: E731
        self.x, self.a, self.b = bf(m, k), bf(slots, r, k, std=k ** -0.5), bf(slots, n, r, std=r ** -0.5)
        self.f32, self.dtype = f32, torch.float32 if f32 else torch.bfloat16
        self.base = bf(m, n).to(self.dtype) if base else None
        self.adapter = torch.tensor(adapter, dtype=torch.int32, device="cuda:0")
        self.ranks = None if ranks is None else torch.tensor(ranks, dtype=torch.int32, device="cuda:0")
        self.scales = torch.rand(slots, generator=g, device="cuda:0") * 2 - 0.7 if scales else None

    def run(self, act="none", work=True, out=None, base="own", **kw):
        import paper_2306_03622_amd as tp
        import torch
        if out is None:
            out = torch.full((self.x.shape[0], self.b.shape[1]), 9.0, dtype=self.dtype, device="cuda:0")
        w = scratch() if work is True else None if work is False else work
        torch.cuda.synchronize()
        tp.tps_lora(self.x, self.a, self.b, self.adapter, out, base=self.base if base == "own" else base, ranks=self.ranks,
                    scales=self.scales, act=act, work=w, **kw)
        torch.cuda.synchronize()
        return out

    def want(self, act="none"):
        d = lambda t: t.double().cpu().numpy()                                                                # noqa: E731
        slots, r, _ = self.a.shape
        ranks = [r] * slots if self.ranks is None else np.clip(self.ranks.cpu().numpy(), 0, r)
        scales = np.ones(slots) if self.scales is None else d(self.scales)
        base = np.zeros((self.x.shape[0], self.b.shape[1])) if self.base is None else d(self.base)
        return lora(d(self.x), d(self.a), d(self.b), self.adapter.cpu().numpy(), base, ranks, scales, act, self.f32)

    def check(self, out, act="none"):
        want, tol = self.want(act)
        off = np.abs(out.double().cpu().numpy() - want)
        assert (off <= tol).all(), (float((off - tol).max()), np.unravel_index((off - tol).argmax(), off.shape))
        log(f"  worst share of the tolerance {float((off / tol).max()):.2f}")


def mixed(m, slots):
    return [(7 * i + i // 5) % slots if i % 7 != 3 else -1 for i in range(m)]


def grouped(m, slots):
    return [i * slots // m for i in range(m)]


# (rows, inputs, outputs, rank, adapters, rows' adapters, ranks, activation, fp32)
CASES = [
    (1, 8, 1, 8, 1, mixed, None, "none", False),
    (1, 768, 768, 8, 4, mixed, None, "none", False),
    (3, 64, 17, 16, 2, mixed, [16, 3], "none", True),
    (16, 4096, 256, 16, 5, mixed, [16, 12, 1, 0, 7], "relu", False),
    (17, 136, 300, 24, 3, grouped, [24, 17, 9], "gelu", True),
    (64, 1024, 1000, 32, 24, mixed, None, "none", False),
    (100, 2048, 1000, 32, 7, grouped, [32, 24, 8, 32, 31, 33, -2], "none", True),
    (33, 40, 515, 128, 6, mixed, [128, 127, 100, 64, 65, 8], "gelu", False),
    (200, 8, 64, 64, 200, grouped, None, "relu", True),
    (700, 256, 136, 48, 3, grouped, [48, 40, 33], "gelu", False),
    (1500, 72, 65, 8, 31, mixed, None, "none", True),
]


@pytest.mark.parametrize("i", range(len(CASES)))
def test_results(i):
    import torch
    m, k, n, r, slots, ids, ranks, act, f32 = CASES[i]
    log(f"{m} rows, {k} -> {n}, {slots} adapters of {r}, {ranks}, {act}, fp32 {f32}")
    s = Setup(300 + i, m, k, n, r, slots, f32, ids(m, slots), ranks)
    for work in (True, False, torch.empty(256 * ((m * r * 4 // 3 + 255) // 256), dtype=torch.uint8, device="cuda:0").fill_(255)):
        s.check(s.run(act, work=work), act)
    s.scales = None
    s.check(s.run(act), act)
    s.base = None
    s.check(s.run(act), act)


def test_rows_without_an_adapter():
    import torch
    for f32 in (False, True):
        s = Setup(1, 40, 64, 100, 8, 3, f32, [-1, 3, 2 ** 31 - 1, -(2 ** 31)] * 10)
        assert bool((s.run() == s.base).all())
        assert bool((s.run("relu") == s.base.clamp(min=0)).all())
        s.base = None
        assert not bool(s.run().any())


def test_in_place_and_layouts():
    import torch
    for f32 in (False, True):
        s = Setup(2, 37, 200, 130, 16, 4, f32, mixed(37, 4), [16, 5, 11, 2])
        want = s.run("gelu")
        s.check(want, "gelu")
        y = s.base.clone()
        assert bool((s.run("gelu", out=y, base=y) == want).all())
        # rows of odd strides and places: 1 element off a 16-byte boundary
        wide = torch.zeros(37, 151, dtype=s.dtype, device="cuda:0")
        wide[:, 3:133] = s.base
        out = torch.full((37, 141), 9.0, dtype=s.dtype, device="cuda:0")
        assert bool((s.run("gelu", out=out[:, 1:131], base=wide[:, 3:133]) == want).all())
        assert bool((out[:, :1] == 9).all()) and bool((out[:, 131:] == 9).all())
        # a base that is the same for all rows
        row = s.base[:1].expand(37, 130)
        got = s.run("gelu", base=row)
        s.base = row.contiguous()
        assert bool((got == s.run("gelu")).all())
        s.x = torch.cat((s.x, s.x), dim=1)[:, :200]
        s.check(s.run("gelu"), "gelu")


def test_one_row_does_not_touch_another():
    # rows, adapters and places behind a rank that hold infinities and NaN
    import torch
    for m, ids in ((24, mixed(24, 5)), (600, grouped(600, 5))):
        s = Setup(3, m, 96, 70, 32, 5, False, ids, [32, 20, 9, 32, 1])
        want = s.run()
        s.a[1, 20:], s.b[1, :, 20:], s.a[2, 9:], s.b[2, :, 9:], s.b[4, :, 1:] = (float("nan"), float("inf"), -float("inf"), float("nan"), float("inf"))
        assert bool((s.run() == want).all())
        s.a[3, 4, 7], s.b[0, 11, 2] = float("inf"), float("nan")
        s.x[5, 3] = float("nan")
        out = s.run()
        odd = ~torch.isfinite(out)
        mine = s.adapter.view(-1, 1)
        expect = (mine == 3).expand_as(odd).clone()
        expect[:, 11] |= mine[:, 0] == 0
        expect[5] = mine[5, 0] >= 0
        assert bool((odd == expect).all())
        assert bool((out[~expect] == want[~expect]).all())
        for act in ("relu", "gelu"):
            assert bool((~torch.isfinite(s.run(act)) | ~expect | (s.run(act) == 0)).all())
            assert bool(torch.isnan(s.run(act)[torch.isnan(out)]).all())


def test_the_same_row_gives_the_same_result_wherever_it_stands():
    import torch
    s = Setup(4, 48, 512, 260, 16, 6, True, mixed(48, 6))
    out = s.run()
    again = s.run()
    assert bool((out == again).all())
    s.x, s.adapter, s.base = s.x[16:17].clone(), s.adapter[16:17].clone(), s.base[16:17].clone()
    s.check(s.run())


def test_adapters_far_apart():
    # a pool whose adapters lie beyond 2^32 bytes
    import torch
    r, k, n = 16, 64, 64
    s = Setup(6, 20, k, n, r, 3, True, mixed(20, 3))
    step = (5 << 30) // 4
    big = torch.zeros(2 * step + r * k + n * r, dtype=torch.bfloat16, device="cuda:0")
    a, b = big.as_strided((3, r, k), (step, k, 1)), big.as_strided((3, n, r), (step, r, 1), storage_offset=r * k)
    a.copy_(s.a)
    b.copy_(s.b)
    want = s.run()
    s.check(want)
    s.a, s.b = a, b
    assert bool((s.run() == want).all())


def test_streams_and_captured_graphs():
    import paper_2306_03622_amd as tp
    import torch
    setups = [Setup(7, 5, 512, 768, 16, 4, False, mixed(5, 4)), Setup(8, 300, 768, 512, 32, 3, True, grouped(300, 3), [32, 7, 20])]
    want, calls = [], []
    for s in setups:
        want.append(s.run())
        s.check(want[-1])
        out, work = torch.zeros_like(want[-1]), scratch()
        calls.append((lambda s=s, out=out, work=work: tp.tps_lora(s.x, s.a, s.b, s.adapter, out, base=s.base, ranks=s.ranks,
                                                                  scales=s.scales, work=work), out))
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


@pytest.mark.parametrize("m,k,n,r,slots", [(1100, 640, 203, 40, 5), (513, 512, 65, 8, 7), (4096, 1024, 70, 64, 2), (600, 520, 131, 24, 19)])
def test_rows_put_in_order(m, k, n, r, slots):
    """Rows that come in order, in turn and at random, few or all of them without an adapter, in place, captured once for all of them."""
    import paper_2306_03622_amd as tp
    import torch
    rng = np.random.default_rng(m)
    orders = [grouped(m, slots), mixed(m, slots), rng.integers(-2, slots + 3, m).tolist(), [slots - 1] * m, [-1] * (m - 1) + [0], [slots] * m]
    s = Setup(9, m, k, n, r, slots, False, orders[0], [max(1, r - 5 * a) for a in range(slots)])
    out, work = s.base.clone(), scratch()

    def call():
        out.copy_(s.base)
        tp.tps_lora(s.x, s.a, s.b, s.adapter, out, base=out, ranks=s.ranks, scales=s.scales, act="relu", work=work)

    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for turn, ids in enumerate(orders + orders[:2]):
        s.adapter.copy_(torch.tensor(ids, dtype=torch.int32))
        want = s.run("relu")
        log(f"order {turn}")
        s.check(want, "relu")
        out.fill_(-3)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert bool((out == want).all()), turn
