"""Every kernel of the attention over a cache and of the adapters, by shapes that the plan gives to each (a CPU test holds the shapes to
their kernels): values against 64 bits, and that a call's scratch is all that it writes beside its result."""
import numpy as np
import pytest

from tests.common import log
from tests.test_gpu_cache_attention import Setup as Attention
from tests.test_gpu_lora import Setup as Lora
from tests.test_gpu_lora import grouped, mixed

pytestmark = pytest.mark.gpu

# (blocks of 16 rows, waves, keys split), new tokens, heads, key/value heads, page, lengths, options: for both dims and both types,
# and those of two waves by (dim, 8 bits)
PAIRS = {
    (64, False): [((1, 2, False), 1, 48, 24, 16, [70, 33, 1] * 3 + [70, 2], {}), ((1, 2, True), 1, 4, 4, 16, [700, 350] * 11, {})],
    (128, False): [((1, 2, False), 1, 48, 24, 16, [70, 33, 1] * 3 + [70, 2], {}), ((1, 2, True), 1, 4, 4, 16, [700, 350] * 11, {})],
    (64, True): [((1, 2, False), 1, 48, 24, 16, [70, 33, 1] * 11, {"window": 200})],
    (128, True): [((1, 2, False), 1, 24, 24, 16, [70, 1] * 11, {})],
}
ATTENTION = [
    ((1, 1, False), 1, 4, 2, 16, [50, 33, 1], {}),
    ((1, 1, False), 3, 4, 1, 32, [2000, 35], {"window": 40, "sinks": 9}),
    ((1, 4, False), 1, 8, 2, 64, [200, 90], {}),
    ((1, 4, True), 2, 8, 1, 16, [5000], {}),
    ((1, 4, True), 1, 4, 2, 128, [3000, 1], {"window": 2000, "sinks": 100}),
    ((2, 4, False), 4, 8, 1, 32, [180, 20], {}),
    ((2, 4, True), 4, 16, 2, 16, [2500, 77], {}),
    ((4, 4, False), 40, 4, 1, 16, [120, 40], {}),
    ((4, 4, True), 33, 4, 2, 64, [4000], {"sinks": 5, "window": 3000}),
]

# (ranks' blocks of 16 and chunks of 32, splits of K or 0 for one launch, several runs, in order first (1) or beside (2)), rows, inputs, outputs, rank,
# adapters, rows' adapters
LORA = [
    ((1, 1, 0, False, 0), 1, 704, 300, 16, 3, mixed),
    ((1, 1, 0, False, 0), 200, 248, 130, 8, 1, grouped),
    ((1, 1, 4, False, 0), 5, 2048, 200, 16, 3, mixed),
    ((2, 1, 1, False, 0), 60, 104, 90, 24, 9, mixed),
    ((2, 1, 1, True, 0), 90, 64, 26000, 32, 5, grouped),
    ((4, 2, 2, False, 0), 33, 1104, 70, 56, 4, mixed),
    ((4, 2, 1, False, 1), 450, 520, 270, 40, 20, mixed),
    ((4, 2, 2, True, 2), 4100, 1032, 2112, 56, 3, grouped),
    ((1, 1, 1, True, 0), 4200, 520, 2112, 16, 1, grouped),       # results past the caches
    ((4, 2, 1, True, 0), 4200, 200, 2112, 64, 1, grouped),
    ((8, 4, 1, True, 0), 4200, 200, 2112, 128, 1, grouped),
    ((1, 1, 1, True, 0), 4200, 520, 2051, 16, 1, grouped),       # as many, whose rows are no whole lines
    ((8, 4, 1, True, 1), 920, 200, 3300, 104, 9, mixed),
    ((8, 4, 2, False, 0), 40, 1032, 66, 128, 2, grouped),
    ((1, 1, 1, False, 2), 777, 520, 131, 16, 7, mixed),
    ((2, 1, 1, False, 2), 1025, 512, 64, 32, 2, mixed),
    ((4, 2, 2, True, 2), 600, 1024, 3000, 64, 3, mixed),
    ((8, 4, 1, False, 2), 8191, 520, 70, 72, 5, mixed),
    ((1, 1, 1, False, 2), 16384, 1024, 64, 8, 7, mixed),             # the most rows beside the first product
    ((4, 2, 1, True, 2), 16383, 1032, 70, 40, 2, grouped),
    ((1, 1, 1, False, 0), 70, 104, 700, 16, 9, mixed),              # adapters of few rows, and of many
    ((2, 1, 1, False, 0), 200, 72, 333, 32, 4, lambda m, slots: [0] * 100 + [1, 2, 3, -1] * 25),
    ((2, 1, 2, False, 0), 40, 1032, 500, 24, 6, grouped),
    ((1, 1, 8, False, 0), 2, 4104, 64, 8, 2, mixed),
]


def guarded(nbytes):
    """Scratch of so many bytes between two stretches that no call may touch."""
    import torch
    whole = torch.full((nbytes + 512,), 77, dtype=torch.uint8, device="cuda:0")
    return whole, whole[256:256 + nbytes]


def untouched(whole):
    return bool((whole[:256] == 77).all()) and bool((whole[-256:] == 77).all())


@pytest.mark.parametrize("dim,e4m3,i", [(d, e, i) for (d, e), more in PAIRS.items() for i in range(len(ATTENTION) + len(more))])
def test_attention(dim, e4m3, i):
    import paper_2306_03622_amd as tp
    import torch
    from tests.test_gpu_cache_rows import dev
    kernel, nq, h, hk, page, lens, kw = (ATTENTION + PAIRS[dim, e4m3])[i]
    log(f"{kernel} {nq} over {lens}, {h} / {hk} heads of {dim}")
    s = Attention(700 + i, len(lens), nq, h, hk, dim, page, lens, e4m3)
    whole, work = guarded(tp.TPO_WORK_BYTES)
    out = torch.full(s.q.shape, 5.0, dtype=torch.bfloat16, device="cuda:0")
    tp.tps_cache_attention(s.cache, dev(s.table), torch.tensor(lens, dtype=torch.int32, device="cuda:0"), s.q, out, work=work, **kw)
    s.check(out, **kw, every=max(1, h // 8))
    assert untouched(whole)
    # scratch that holds two parts of the keys, and no more
    nbytes = 2 * len(lens) * nq * h * (dim + 2) * 4 // 256 * 256 + 256
    whole, work = guarded(nbytes)
    out.fill_(5.0)
    tp.tps_cache_attention(s.cache, dev(s.table), torch.tensor(lens, dtype=torch.int32, device="cuda:0"), s.q, out, work=work, **kw)
    s.check(out, **kw, every=max(1, h // 8))
    assert untouched(whole)


@pytest.mark.parametrize("f32", [False, True])
@pytest.mark.parametrize("i", range(len(LORA)))
def test_adapters(i, f32):
    import paper_2306_03622_amd as tp
    kernel, m, k, n, r, slots, ids = LORA[i]
    log(f"{kernel} {m} rows, {k} -> {n}, {slots} adapters of {r}")
    s = Lora(800 + i, m, k, n, r, slots, f32, ids(m, slots), [max(1, r - 3 * (a % 4)) for a in range(slots)])
    for nbytes in (tp.TPO_WORK_BYTES, m * (r + 2) * 4 // 256 * 256 + 256, m * r * 4 // 256 * 256 + 256):
        whole, work = guarded(nbytes)
        s.check(s.run("gelu", work=work), "gelu")
        assert untouched(whole)
