"""Attention over pages, plain and of trees, for few rows behind long lists and 1 to 3 kv heads: lists are cut there into as many parts as a
chip full of items takes.  Against the definition in 64 bits, with a pattern behind the workspace that has to stay, and the number of
work items as the host's view of the rules has it."""
import pytest

import drafts_model as M
import paper_2502_02175_amd as V
import test_gpu_attend as plain
import test_gpu_tree as trees_of
from pages_model import OK, PAGE
from test_gpu_attend import DEV, Cache, i32, queries

pytestmark = pytest.mark.gpu
BEHIND = 1 << 20


def passes(c, p, seqs, pos, q, stem, trees=None):
    """One pass -> out, columns of a block; the plan's items and the pattern behind the workspace looked at."""
    import torch
    n, T, hq, _ = q.shape
    size = (V.vlac_attend_workspace_bytes if trees is None else V.vlac_attend_tree_workspace_bytes)(p, n, T, hq)
    room = torch.full((size + BEHIND,), 0x5A, dtype=torch.uint8, device=DEV)
    ws, out = room[:size], torch.full(q.shape, 7.0, dtype=c.dt, device=DEV)
    if trees is None:
        V.vlac_attend_plan(p, i32(seqs), i32(pos), n, T, hq, None, ws)
    else:
        V.vlac_attend_tree_plan(p, i32(seqs), i32(pos), n, T, hq, None, i32(trees), None, ws)
    cols, (items, items_room), (parts, parts_room) = V.vlac_plan_attention(p, T, hq, pos, None, [stem] * n)
    assert ws[:4].view(torch.int32).item() == items <= items_room and parts <= parts_room
    if trees is None:
        V.vlac_attend_shared(p, 0, n, T, hq, q, out, ws)
    else:
        V.vlac_attend_tree(p, 0, n, T, hq, q, out, ws)
    assert bool((room[size:] == 0x5A).all())
    assert V.vlac_pages_check(p, check=False) == OK
    return out, cols


def check(c, p, seqs, pos, q, stem, trees=None, some=None):
    some = list(range(len(seqs))) if some is None else some
    out, cols = passes(c, p, seqs, pos, q, stem, trees)
    at = [seqs[i] for i in some], [pos[i] for i in some], q[some]
    want, tol = plain.definition(c, *at) if trees is None else trees_of.definition(c, *at, [trees[i] for i in some])
    err = (out[some].double() - want).abs()
    assert bool((err <= tol).all()), "%.3g over the bound" % float((err / tol).max())
    return cols


@pytest.mark.parametrize("hq,hkv,hd,operand", [(1, 1, 64, 1), (8, 1, 128, 0), (16, 1, 64, 0), (4, 2, 64, 1), (12, 2, 128, 1), (3, 3, 128, 0), (9, 3, 64, 1)])
@pytest.mark.parametrize("n", [5, 48, 171])
@pytest.mark.parametrize("T", [1, 2])
def test_groups_behind_long_lists(hq, hkv, hd, operand, n, T):
    c = Cache(hkv, hd, operand, seed=hq + n)
    stem = 133
    base = [c._new(PAGE) for _ in range(stem)]
    pos = [stem * PAGE + i % 40 for i in range(n)]
    seqs = [c.sequence(x + T, base) for x in pos]
    p, q = c.pool(), queries(c, n, T, hq)
    some = list(range(0, n, 7)) + [n - 1]
    check(c, p, seqs, pos, q, stem, some=some)
    check(c, p, seqs, pos, q, stem, [M.some_tree(i, T, ("random", "holes", "roots")[i % 3]) for i in range(n)], some)


def test_a_step_of_a_small_decoder():
    """24 candidates, 8 heads on one kv head, 33000 positions."""
    c = Cache(1, 128, 0, seed=24)
    stem = 33000 // PAGE
    base = [c._new(PAGE) for _ in range(stem)]
    pos = [33000 + i % 5 for i in range(24)]
    seqs = [c.sequence(x + 1, base) for x in pos]
    assert check(c, c.pool(), seqs, pos, queries(c, 24, 1, 8), stem) == 32


@pytest.mark.parametrize("hq,hkv,n,stem", [(1, 1, 129, 32000), (1, 1, 171, 6000), (3, 3, 43, 32000), (2, 2, 43, 9200), (2, 1, 86, 9200)])
@pytest.mark.parametrize("tree", [False, True])
def test_the_most_parts(hq, hkv, n, stem, tree):
    """Up to a million positions that all entries share (a thousand pages, again and again): as many parts as the workspace has room for."""
    c = Cache(hkv, 64, 1, seed=n)
    base = [c._new(PAGE) for _ in range(1000)]
    base = (base * (stem // 1000 + 1))[:stem]
    pos = [stem * PAGE + i % 30 for i in range(n)]
    seqs = [c.sequence(x + 1, base) for x in pos]
    assert check(c, c.pool(), seqs, pos, queries(c, n, 1, hq), stem, [[-1]] * n if tree else None, [0, 1, n // 2, n - 1]) == 32
