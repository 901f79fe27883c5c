"""Every kernel of tps_cache_append and tps_cache_read, by shapes that the plan gives to each (a CPU test holds the shapes to their
kernels): every place of the pool, every row read back, and what neither may touch."""
import numpy as np
import pytest

from tests.common import log
from tests.serve_common import e4m3_rows
from tests.test_gpu_cache_rows import bits, dev, make_cache, table_of

pytestmark = pytest.mark.gpu

# (rows in each place of a workgroup, workgroups side by side for a token, rows side by side in one), dim, heads, page, rows, lengths, new ones
ROWS = [
    ((1, 1, 2), 64, 12, 16, 9, [40, 9, 3], [9, 0, 5]),
    ((1, 1, 3), 128, 5, 32, 70, [70, 200], None),
    ((1, 2, 1), 64, 33, 16, 5, [33, 5, 70], [5, 2, 1]),
    ((1, 2, 1), 128, 17, 64, 7, [7, 100], [6, 7]),
    ((1, 3, 1), 128, 40, 16, 2, [2, 19], None),
    ((2, 1, 2), 64, 12, 16, 413, [413, 500, 1000, 77, 414], [413, 412, 1, 77, 0]),
    ((2, 1, 16), 64, 2, 128, 3301, [3301, 4000, 3301, 9000, 3500], None),
    ((2, 1, 3), 128, 5, 16, 617, [617, 619, 1200, 616, 700], [617, 1, 616, 616, 615]),
    ((2, 1, 2), 128, 8, 64, 701, [701, 900, 703], None),
    ((2, 2, 1), 64, 33, 32, 261, [261, 300], [260, 261]),
    ((2, 2, 1), 128, 17, 16, 261, [300, 261], None),
    ((2, 3, 1), 128, 40, 16, 173, [173, 180], [173, 90]),
]


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("i", range(len(ROWS)))
def test_rows(i, e4m3):
    import paper_2306_03622_amd as tp
    import torch
    kernel, dim, heads, page, rows, kv_lens, q_lens = ROWS[i]
    log(f"{kernel} {rows} rows of {heads} x {dim}, pages of {page}, {kv_lens}, {q_lens}")
    rng = np.random.default_rng(80 + i)
    batch, columns = len(kv_lens), max((n + page - 1) // page for n in kv_lens)
    pages = batch * columns + 2
    table = table_of(rng, batch, columns, pages)
    cache, (pk, pv), exps = make_cache(pages, page, heads, dim, e4m3, "padded" if i % 2 else "tokens")
    torch.manual_seed(i)
    new = torch.randn(2, batch, rows, heads, dim, device="cuda:0").mul_(
        torch.randint(-20, 20, (2, batch, rows, heads, 1), device="cuda:0").float().exp2()).to(torch.bfloat16)
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda:0")          # noqa: E731
    tb, kl, ql = dev(table), i32(kv_lens), None if q_lens is None else i32(q_lens)
    tp.tps_cache_append(cache, tb, kl, new[0], new[1], q_lens=ql)
    out = torch.full((2, batch, rows, heads, dim), 7.0, dtype=torch.bfloat16, device="cuda:0")
    tp.tps_cache_read(cache, tb, kl, out[0], out[1], q_lens=ql)
    torch.cuda.synchronize()
    x = new.double().cpu().numpy()
    codes, ex, values = e4m3_rows(x) if e4m3 else (bits(new), None, x)
    want = [np.full((pages, page, heads, dim), 3 if e4m3 else 0x4040, dtype=codes.dtype) for _ in "kv"]
    wex = np.full((pages, 2, heads, page), 9, dtype=np.uint8)
    back = np.full(out.shape, 7.0)
    for b in range(batch):
        qn = rows if q_lens is None else q_lens[b]
        first = max(0, qn - kv_lens[b])             # (rows in front of token 0 are in no page)
        pos = np.arange(kv_lens[b] - qn + first, kv_lens[b])
        p, at = table[b, pos // page], pos % page
        back[:, b, :first] = 0
        for n in range(2):
            want[n][p, at], back[n, b, first:qn] = codes[n, b, first:qn], values[n, b, first:qn]
            if e4m3:
                wex[p, n, :, at] = ex[n, b, first:qn]
    for got, w in zip((pk, pv), want):
        assert np.array_equal(got.cpu().numpy() if e4m3 else bits(got), w)
    if e4m3:
        assert np.array_equal(exps.cpu().numpy(), wex)
    assert np.array_equal(out.double().cpu().numpy(), back)
