"""The serving operators one after another as a decoder's layer for many tenants uses them: 4-bit projections that all share, each request's
own adapters beside them, a paged cache that grows by the new tokens. Against the same layer in 64 bits, on two streams at
once, and captured."""
import numpy as np
import pytest

from tests.common import log
from tests.ops_common import bf16, w4_plain, w4_tolerance
from tests.serve_common import Pool, cache_attention, e4m3_rows, e4m3_values, lora, seen
from tests.test_gpu_linear_w4 import bf_tensor, scratch, weight

pytestmark = pytest.mark.gpu

HEADS, KV_HEADS, DIM, PAGE, GROUP, RANK, SLOTS = 8, 2, 64, 16, 64, 16, 3
WIDTH = HEADS * DIM
NEW = (HEADS + 2 * KV_HEADS) * DIM
LENS = [301, 2, 77, 640]                               # with the new tokens
TENANTS = [1, -1, 0, 1]
WINDOW, SINKS = 500, 3


class Layer:
    """x + adapted(attention(adapted(x Wqkv)) Wo): tokens new ones for each sequence, the last of LENS."""

    def __init__(self, seed, tokens, e4m3):
        import paper_2306_03622_amd as tp
        import torch
        rng = np.random.default_rng(seed)
        g = torch.Generator(device="cuda:0")
        g.manual_seed(seed)
        self.tokens, self.e4m3, batch = tokens, e4m3, len(LENS)
        self.plain = [w4_plain(rng, n, WIDTH, GROUP) for n in (NEW, WIDTH)]
        self.w = [weight(c, b, GROUP) for c, b, _ in self.plain]
        r = lambda *s, std=1.0: (torch.randn(*s, generator=g, device="cuda:0") * std).to(torch.bfloat16)       # noqa: E731
        self.down = [r(SLOTS, RANK, WIDTH, std=WIDTH ** -0.5) for _ in self.w]
        self.up = [r(SLOTS, n, RANK, std=RANK ** -0.5) for n in (NEW, WIDTH)]
        self.x_np = bf16(rng.standard_normal((batch * tokens, WIDTH)) * 0.02)
        self.x = bf_tensor(self.x_np)
        columns = max((n + PAGE - 1) // PAGE for n in LENS)
        pages = batch * columns + 2
        self.table_np = rng.permutation(pages)[:batch * columns].reshape(batch, columns).astype(np.int32)
        self.table = torch.from_numpy(self.table_np).to("cuda:0")
        dtype = torch.float8_e4m3fn if e4m3 else torch.bfloat16
        self.k, self.v = ((r(pages, PAGE, KV_HEADS, DIM).float() * (60 if e4m3 else 1)).to(dtype) for _ in "kv")
        self.exps = torch.full((pages, 2, KV_HEADS, PAGE), 121, dtype=torch.uint8, device="cuda:0") if e4m3 else None
        self.cache = tp.PagedCache(self.k, self.v, self.exps)
        i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda:0")                                 # noqa: E731
        self.lens, self.ranks, self.scales = i32(LENS), i32([RANK, 9, 3]), torch.tensor([1.0, -0.5, 2.0], device="cuda:0")
        self.adapter = i32([t for t in TENANTS for _ in range(tokens)])
        self.shared, self.mid = r(batch * tokens, NEW), r(batch * tokens, NEW)
        self.att = r(batch, tokens, HEADS, DIM)
        self.sum, self.out = r(batch * tokens, WIDTH), r(batch * tokens, WIDTH)
        self.work = scratch()

    def step(self):
        import paper_2306_03622_amd as tp
        lo = {"ranks": self.ranks, "scales": self.scales, "work": self.work}
        tp.tpo_linear_w4(self.x, self.w[0], self.shared, work=self.work)
        tp.tps_lora(self.x, self.down[0], self.up[0], self.adapter, self.mid, base=self.shared, **lo)
        heads = self.mid.view(len(LENS), self.tokens, HEADS + 2 * KV_HEADS, DIM)
        tp.tps_cache_append(self.cache, self.table, self.lens, heads[:, :, HEADS:HEADS + KV_HEADS], heads[:, :, HEADS + KV_HEADS:])
        tp.tps_cache_attention(self.cache, self.table, self.lens, heads[:, :, :HEADS], self.att, window=WINDOW, sinks=SINKS, work=self.work)
        att = self.att.view(-1, WIDTH)
        tp.tpo_linear_w4(att, self.w[1], self.sum, res=self.x, work=self.work)
        self.out.copy_(self.sum)
        tp.tps_lora(att, self.down[1], self.up[1], self.adapter, self.out, base=self.out, **lo)             # in place

    def results(self):
        out = [self.shared, self.mid, self.att, self.sum, self.out, self.k, self.v]
        return [t.float() for t in out] + ([self.exps.float()] if self.e4m3 else [])

    def clear(self):
        for t in (self.shared, self.mid, self.att, self.sum, self.out):
            t.fill_(-3)

    def pool(self):
        import torch
        got = []
        for n, t in enumerate((self.k, self.v)):
            if self.e4m3:
                x = e4m3_values()[t.view(torch.uint8).cpu().numpy()]
                got.append(x * 2.0 ** (self.exps[:, n].cpu().numpy().astype(np.float64) - 127).transpose(0, 2, 1)[..., None])
            else:
                got.append(t.double().cpu().numpy())
        return got


@pytest.mark.parametrize("tokens,e4m3", [(1, False), (1, True), (2, False), (2, True)])
def test_against_64_bits(tokens, e4m3):
    import torch
    layer = Layer(5 + tokens, tokens, e4m3)
    before = layer.pool()
    layer.step()
    torch.cuda.synchronize()
    log("step done")
    d = lambda t: t.double().cpu().numpy()                                                                 # noqa: E731
    # each stage from the values the stage before really gave, so that a stage's own rounding is all there is
    shared, mid, att, total, out = (d(t) for t in (layer.shared, layer.mid, layer.att, layer.sum, layer.out))
    flat = att.reshape(-1, WIDTH)
    ids, ranks, scales = layer.adapter.cpu().numpy(), layer.ranks.cpu().numpy(), d(layer.scales)
    for i, (x, got, res, adapted) in enumerate(((layer.x_np, shared, 0, mid), (flat, total, layer.x_np, out))):
        want = x @ layer.plain[i][2].T + res
        assert (np.abs(got - want) <= w4_tolerance(x, layer.plain[i][2], want, False)).all()
        want, tol = lora(x, d(layer.down[i]), d(layer.up[i]), ids, got, ranks, scales, "none", False)
        assert (np.abs(adapted - want) <= tol).all()
    heads = mid.reshape(len(LENS), tokens, HEADS + 2 * KV_HEADS, DIM)
    for b, n in enumerate(LENS):
        for i in range(tokens):
            page, at = layer.table_np[b, (n - tokens + i) // PAGE], (n - tokens + i) % PAGE
            for j, pool in enumerate(before):
                new = heads[b, i, HEADS + j * KV_HEADS:HEADS + (j + 1) * KV_HEADS]
                pool[page, at] = e4m3_rows(new)[2] if e4m3 else new
    for pool, got in zip(before, layer.pool()):
        assert np.array_equal(pool, got)
    pool = Pool(*before, layer.table_np, PAGE)
    for b, n in enumerate(LENS):
        k, v, _ = pool.sequence(b, n)
        m = seen(tokens, n, WINDOW, SINKS)
        for h in range(HEADS):
            g = h // (HEADS // KV_HEADS)
            want, tol = cache_attention(heads[b, :, h], k[:, g], v[:, g], m, DIM ** -0.5)
            assert (np.abs(att[b, :, h] - want) <= tol).all(), (b, h)


def test_two_streams_at_once_and_graphs():
    import torch
    layers = [Layer(21, 1, False), Layer(22, 2, True)]
    want = []
    for l in layers:
        l.step()
        torch.cuda.synchronize()
        want.append([t.clone() for t in l.results()])
    same = lambda l, w: all(bool((a == b).all()) for a, b in zip(l.results(), w))                           # noqa: E731
    streams = [torch.cuda.Stream(device="cuda:0") for _ in layers]
    for l in layers:
        l.clear()
    torch.cuda.synchronize()
    for _ in range(20):                                # turn by turn, nothing waits in between
        for l, s in zip(layers, streams):
            with torch.cuda.stream(s):
                l.step()
    torch.cuda.synchronize()
    log("two streams")
    assert all(same(l, w) for l, w in zip(layers, want))
    graphs = []
    for l in layers:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            l.step()
        graphs.append(g)
    for turn in range(4):
        for l in layers:
            l.clear()
        torch.cuda.synchronize()
        for g, s in zip(graphs, streams):              # replays that overlap: each graph has scratch of its own
            with torch.cuda.stream(s):
                g.replay()
        torch.cuda.synchronize()
        log(f"replay {turn}")
        assert all(same(l, w) for l, w in zip(layers, want))
