"""tps_lora with scratch that holds the inner sums of a part of the rows: values, in place, a base for all rows, captured."""
import pytest

from tests.common import log
from tests.test_gpu_lora import Setup, grouped, mixed
from tests.test_gpu_serve_variants import guarded, untouched

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("f32", [False, True])
@pytest.mark.parametrize("m,k,n,r,slots,ids,rows", [
    (2050, 72, 300, 16, 3, mixed, 1024),            # a last part of two rows
    (3000, 520, 515, 40, 20, mixed, 1100),          # put in order first
    (2500, 1032, 260, 8, 5, mixed, 1300),           # beside the first product
    (4100, 64, 700, 128, 1, grouped, 1024),
    (9000, 64, 130, 64, 2, grouped, 4200),
])
def test_parts(m, k, n, r, slots, ids, rows, f32):
    import paper_2306_03622_amd as tp
    import torch
    log(f"{m} rows in parts of up to {rows}, {k} -> {n}, {slots} adapters of {r}, fp32 {f32}")
    s = Setup(1200 + m, m, k, n, r, slots, f32, ids(m, slots), [max(1, r - 3 * a) for a in range(slots)])
    size = 4 * rows * (r + 2)
    whole, work = guarded((size + 255) // 256 * 256)
    want = s.run("relu", work=work)
    s.check(want, "relu")
    assert untouched(whole)
    out = s.base.clone()
    assert torch.equal(s.run("relu", work=work, out=out, base=out), want)
    # rows of a stride of their own, results among others
    wide = torch.full((m, n + 9), 3.0, dtype=s.dtype, device="cuda:0")
    wide[:, 4:4 + n] = s.base
    s.x = torch.cat((s.x, s.x), dim=1)[:, :k]
    assert torch.equal(s.run("relu", work=work, out=wide[:, 4:4 + n], base=wide[:, 4:4 + n]), want)
    assert bool((wide[:, :4] == 3).all()) and bool((wide[:, 4 + n:] == 3).all())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out.copy_(s.base)
        tp.tps_lora(s.x, s.a, s.b, s.adapter, out, base=out, ranks=s.ranks, scales=s.scales, act="relu", work=work)
    for _ in range(3):
        out.fill_(-3)
        work.fill_(255)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)
    # one row for all of them
    row = s.base[:1].expand(m, n)
    got = s.run("relu", work=work, base=row)
    s.base = row.contiguous()
    s.check(got, "relu")


def test_a_row_gives_the_same_bits_in_every_part():
    # (the last part has two rows of long sums: by itself its plan would split them, and add in another order)
    import torch
    m, k, n, r, slots = 2050, 2064, 300, 16, 3
    s = Setup(1300, m, k, n, r, slots, True, mixed(m, slots))
    _, work = guarded(4 * 1024 * (r + 2))
    x, adapter, base, want = s.x, s.adapter, s.base, s.run(work=work)
    for p in (torch.arange(m - 1, -1, -1, device="cuda:0"), torch.roll(torch.arange(m, device="cuda:0"), 700)):
        s.x, s.adapter, s.base = x[p].contiguous(), adapter[p].contiguous(), base[p].contiguous()
        assert torch.equal(s.run(work=work), want[p])
