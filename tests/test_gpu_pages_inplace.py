"""The positions of an extension written over the list of its sequences."""
import pytest

import paper_2502_02175_amd as V
from test_gpu_pages import Both, i32

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n", [5, 256, 300, 1500])
def test_positions_over_the_list(n):
    b = Both(4 * n + 9, 2 * n, 3)
    for turn in range(3):
        seqs = [2 * ((7 * i + turn) % n) for i in range(n)]
        seqs[-1] = seqs[0]                                       # (listed twice: ignored)
        x = i32(seqs)
        V.vlac_pages_extend(b.p, x, n, 20, x)
        assert x.tolist() == b.m.extend(seqs, 20), turn
        b.same("turn %d" % turn)
    odd = [2 * i + 1 for i in range(n)]
    b.fork([0] * n, odd)
    b.extend(odd, 9)                                              # (no mark of an earlier call is left)
    b.extend(list(range(n)), 1)
    b.same("afterwards")
