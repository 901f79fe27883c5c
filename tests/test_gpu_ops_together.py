"""The operators one after another as a decoder's layer uses them, for single tokens over a growing cache: against the same
layer in 64 bits, on two streams at once, and captured."""
import numpy as np
import pytest

from tests.common import log
from tests.ops_common import attention, bf16, seen, w4_plain, w4_tolerance
from tests.test_gpu_linear_w4 import bf_tensor, scratch, weight

pytestmark = pytest.mark.gpu

HEADS, KV_HEADS, DIM, BATCH, ROOM, GROUP = 8, 2, 64, 3, 700, 64
WIDTH = HEADS * DIM
KEEP = {"causal": True, "window": (500, 0), "sinks": 3}


class Layer:
    """x + attention(x Wqkv) Wo, new keys and values written into the cache at each sequence's length."""

    def __init__(self, seed):
        import torch
        rng = np.random.default_rng(seed)
        self.plain = [w4_plain(rng, n, WIDTH, GROUP) for n in ((HEADS + 2 * KV_HEADS) * DIM, WIDTH)]
        self.qkv, self.o = (weight(c, b, GROUP) for c, b, _ in self.plain)
        self.cache_np = bf16(rng.standard_normal((2, BATCH, ROOM, KV_HEADS, DIM)))
        self.cache = bf_tensor(self.cache_np)
        self.x_np = bf16(rng.standard_normal((BATCH, WIDTH)) * 0.02)
        self.x = bf_tensor(self.x_np)
        self.mid = torch.zeros(BATCH, (HEADS + 2 * KV_HEADS) * DIM, dtype=torch.bfloat16, device="cuda:0")
        self.att = torch.zeros(BATCH, 1, HEADS, DIM, dtype=torch.bfloat16, device="cuda:0")
        self.out = torch.zeros(BATCH, WIDTH, dtype=torch.bfloat16, device="cuda:0")
        self.lens = torch.tensor([640, 1, 77], dtype=torch.int32, device="cuda:0")       # with the new token
        self.at = self.lens.long() - 1
        self.rows = torch.arange(BATCH, device="cuda:0")
        self.work = scratch()

    def step(self):
        import paper_2306_03622_amd as tp
        tp.tpo_linear_w4(self.x, self.qkv, self.mid, work=self.work)
        heads = self.mid.view(BATCH, HEADS + 2 * KV_HEADS, DIM)
        self.cache[0].index_put_((self.rows, self.at), heads[:, HEADS:HEADS + KV_HEADS])
        self.cache[1].index_put_((self.rows, self.at), heads[:, HEADS + KV_HEADS:])
        tp.tpo_attention(heads[:, None, :HEADS], self.cache[0], self.cache[1], self.att, kv_lens=self.lens, work=self.work, **KEEP)
        tp.tpo_linear_w4(self.att.view(BATCH, WIDTH), self.o, self.out, res=self.x, work=self.work)

    def clear(self):
        for t in (self.mid, self.att, self.out):
            t.fill_(-3)


def test_against_64_bits():
    import torch
    layer = Layer(5)
    layer.step()
    torch.cuda.synchronize()
    # each stage from the values the stage before really gave, so that a stage's own rounding is all there is
    mid, att, out = (t.double().cpu().numpy() for t in (layer.mid, layer.att, layer.out))
    wq, wo = (w for _, _, w in layer.plain)
    for got, x, w, res in ((mid, layer.x_np, wq, 0), (out, att.reshape(BATCH, WIDTH), wo, layer.x_np)):
        want = x @ w.T + res
        assert (np.abs(got - want) <= w4_tolerance(x, w, want, False)).all()
    heads = mid.reshape(BATCH, HEADS + 2 * KV_HEADS, DIM)
    for b, n in enumerate([640, 1, 77]):
        k, v = layer.cache_np[0, b].copy(), layer.cache_np[1, b].copy()
        k[n - 1], v[n - 1] = heads[b, HEADS:HEADS + KV_HEADS], heads[b, HEADS + KV_HEADS:]
        m = seen(1, n, True, 500, 0, 3)
        for h in range(HEADS):
            g = h // (HEADS // KV_HEADS)
            want, tol = attention(heads[b, h:h + 1], k[:n, g], v[:n, g], m, DIM ** -0.5)
            assert (np.abs(att[b, :, h] - want) <= tol).all(), (b, h)


def test_two_streams_at_once_and_graphs():
    import torch
    layers = [Layer(21), Layer(22)]
    want = []
    for l in layers:
        l.step()
        torch.cuda.synchronize()
        want.append([t.clone() for t in (l.mid, l.att, l.out)])
    same = lambda l, w: all(bool((a == b).all()) for a, b in zip((l.mid, l.att, l.out), w))
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
