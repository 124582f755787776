"""As many heads as a call may have, and as many positions as a sequence may."""
import pytest

import paper_2502_02175_amd as V
from pages_model import OK
from test_gpu_attend import Cache, compare, queries

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("hq,hkv,hd,operand,n,T", [(1024, 1, 64, 1, 3, 1), (1024, 1024, 64, 0, 2, 1), (1024, 8, 128, 1, 2, 3),
                                                   (1000, 125, 64, 1, 3, 2), (1023, 3, 128, 0, 1, 2)])
@pytest.mark.parametrize("columns", [0, 80])
def test_many_heads(hq, hkv, hd, operand, n, T, columns):
    c = Cache(hkv, hd, operand, seed=hq + hkv)
    base = [c._new(32) for _ in range(2)]
    pos = [64 + 9 * i for i in range(n)]
    seqs = [c.sequence(x + T, base) for x in pos]
    if columns:                                                # (a table with room for long lists)
        c.sequence(32 * columns, base * (columns // 2))
    p = c.pool()
    compare(c, p, seqs, pos, queries(c, n, T, hq))
    assert V.vlac_pages_check(p, check=False) == OK


@pytest.mark.parametrize("hq,n", [(1, 1), (8, 6)])
def test_the_longest_sequence(monkeypatch, hq, n):
    """2^20 positions: 32768 pages, each of 1024 pages 32 times."""
    make = V.new_pages
    monkeypatch.setattr(V, "new_pages", lambda *a: make(*a[:6], min(a[6], 32768), a[7]))
    c = Cache(1, 64, 1, seed=n)
    base = [c._new(32) for _ in range(1024)]
    length = 1 << 20
    seqs = [c.sequence(length, base * 31 + base[:1024 - i]) for i in range(n)]
    p = c.pool()
    compare(c, p, seqs, [length - 1] * n, queries(c, n, 1, hq))
    compare(c, p, seqs, [length - 1] * n, queries(c, n, 1, hq), list(range(n)))
    assert V.vlac_pages_check(p, check=False) == OK
