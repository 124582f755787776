"""Tables and lengths that the caller has broken: what does not fit is skipped and reported, nothing is read or written
through it, and the rest of the call goes on."""
import pytest

import paper_2502_02175_amd as V
from pages_model import E_RANGE, OK
from test_gpu_pages import Both, i32

pytestmark = pytest.mark.gpu
FAR = (-1, 70, 2 ** 31 - 1, -2 ** 31)   # of 70 pages


def made():
    """Sequences 0 and 1 of 75 positions (pages 0 1 2 and 3 4 5), 2 a fork of 0 (0 1 6)."""
    b = Both(70, 6, 5)
    b.extend([0, 1], 75)
    b.fork([0], [2])
    b.same()
    return b


def state(b):
    return b.refs.tolist(), b.table.tolist(), b.len.tolist()


def reported(b):
    assert V.vlac_pages_check(b.p, check=False) == E_RANGE
    assert V.vlac_pages_check(b.p, check=False) == OK


@pytest.mark.parametrize("bad", FAR)
def test_release_skips_an_entry_that_is_no_page(bad):
    b = made()
    b.table[1, 1] = bad
    V.vlac_pages_free(b.p, i32([1, 0]), 2)
    refs, table, length = state(b)
    assert refs[:8] == [1, 1, 0, 0, 1, 0, 1, 0] and length[:3] == [0, 0, 75] and table[1] == table[0] == [-1] * 5
    reported(b)
    b = made()
    b.table[1, 1] = bad
    V.vlac_pages_fork(b.p, i32([0]), i32([1]), 1)           # (a destination is released)
    refs, table, length = state(b)
    assert table[1] == [0, 1, 3, -1, -1] and refs[:8] == [3, 3, 1, 1, 1, 0, 1, 0] and length[1] == 75
    reported(b)


@pytest.mark.parametrize("bad", FAR)
@pytest.mark.parametrize("deep", [False, True])
@pytest.mark.parametrize("at", [0, 2])
def test_fork_of_a_source_with_an_entry_that_is_no_page(bad, deep, at):
    b = made()
    b.table[1, at] = bad
    before = b.words.clone()
    V.vlac_pages_fork(b.p, i32([1, 0]), i32([3, 4]), 2, deep)
    refs, table, length = state(b)
    assert length[3:5] == [75, 75]
    fresh = table[4] if deep else [table[4][2]]
    for p, q in zip(fresh, (0, 1, 2) if deep else (2,)):
        assert p >= 7 and refs[p] == 1 and bool((b.words[p] == q).all())
    held = set(p for p in table[3] + table[4] if 0 <= p < 70)
    rest = [p for p in range(70) if p not in held]
    assert bool((b.words[rest] == before[rest]).all())
    reported(b)


@pytest.mark.parametrize("bad", [70, 2 ** 31 - 1, -1, -2 ** 31])
def test_compact_leaves_an_entry_that_is_no_page(bad):
    b = made()
    V.vlac_pages_free(b.p, i32([1]), 1)
    b.table[2, 1] = bad
    live = i32([-7])
    V.vlac_pages_compact(b.p, live)
    refs, table, length = state(b)
    assert live.tolist() == [4] and table[0][:3] == [0, 1, 2] and table[2][:3] == [0, bad, 3] and refs[:5] == [2, 2, 1, 1, 0]
    reported(b)


@pytest.mark.parametrize("bad", [-1, 161, 2 ** 31 - 1, -2 ** 31])
def test_a_length_out_of_range_is_left_as_it_is(bad):
    b = made()
    b.len[1] = bad
    before = state(b)
    V.vlac_pages_free(b.p, i32([1, 1]), 2)
    assert state(b) == before
    reported(b)
    V.vlac_pages_fork(b.p, i32([1, 0]), i32([3, 1]), 2)
    pos = i32([-7])
    V.vlac_pages_extend(b.p, i32([1]), 1, 3, pos)
    assert state(b) == before and pos.tolist() == [-1]
    reported(b)
    V.vlac_pages_free(b.p, i32([0, 2]), 2)
    assert V.vlac_pages_check(b.p, check=False) == OK
    live = i32([-7])
    V.vlac_pages_compact(b.p, live)                            # (moves its pages, and cannot say so in its row)
    assert live.tolist() == [3] and b.table[1].tolist() == [3, 4, 5, -1, -1] and b.len[1] == bad
    reported(b)


@pytest.mark.parametrize("bad", FAR)
@pytest.mark.parametrize("at", [0, 2])
@pytest.mark.parametrize("columns", [4, 80])
def test_attention_past_an_entry_that_is_no_page(bad, at, columns):
    """Among the pages of all (0) and among a sequence's own (2); short tables, and some with room for long lists."""
    import torch
    from test_gpu_attend import Cache, definition, queries, run
    c = Cache(2, 64, 1, seed=3)
    base = [c._new(32) for _ in range(2)]
    pos = [70, 75, 66]
    seqs = [c.sequence(x + 2, base) for x in pos]
    p = c.pool()
    wide = torch.full((p.max_seqs, columns), -1, dtype=torch.int32, device="cuda:0")
    wide[:, :p.max_pages] = p.tensors[2]
    p = V.pages(1, 2, 64, 1, p.tensors[0], p.tensors[1], wide, p.tensors[3])
    p.tensors[2][1, at] = bad
    q = queries(c, 3, 2, 4)
    out = run(p, c, seqs, pos, q, [0, 1, 2])
    want, tol = definition(c, seqs, pos, q)
    fine = [0, 2]
    assert bool(((out.double() - want).abs() <= tol)[fine].all())
    reported(type("", (), {"p": p}))
    p.tensors[2][:3, 0] = bad                                 # the same in all: a common page
    run(p, c, seqs, pos, q, [0, 0, 0])
    reported(type("", (), {"p": p}))
