"""Attention over a table that has room for more tokens than a call can have: the default bound on the lengths stays one that a call takes."""
import pytest

from paper_2306_03622_amd import serve as S
from tests.test_serve_host import Device, a_cache, attention_args, bf, calls, i32, on  # noqa: F401  (calls: a fixture)

torch = pytest.importorskip("torch")
MOST = (1 << 30) - 1


@pytest.mark.parametrize("columns,bound", [(262143, 262143 * 4096), (262144, MOST), (600000, MOST)])
def test_the_default_bound(columns, bound, calls):  # noqa: F811
    import paper_2306_03622_amd as tp
    k, v = (on(torch.zeros(1, 4096, 2, 64, dtype=torch.bfloat16)) for _ in "kv")
    table = on(torch.zeros(1, columns, dtype=torch.int32))
    tp.tps_cache_attention(tp.PagedCache(k, v), table, i32(5), bf(1, 1, 6, 64), bf(1, 1, 6, 64))
    a = S.tps_cache_attention_args.from_buffer_copy(calls.made[-1][0])
    assert (a.kv_len, a.max_pages) == (bound, columns)


def test_that_bound_is_the_most_that_a_call_takes():
    # (refused for its work, which is looked at behind the lengths; one more is refused for the lengths)
    from tests.test_serve_host import _status
    assert "work" in _status("tps_cache_attention", attention_args(kv_len=MOST, work=0x7010))[1]
    assert "kv_len" in _status("tps_cache_attention", attention_args(kv_len=MOST + 1, work=0x7010))[1]
