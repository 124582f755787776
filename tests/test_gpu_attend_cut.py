"""When the plan cuts lists into parts: not where the blocks of many groups fill the chip while the longest list runs.  The first word
of a workspace is the number of work items that the plan left in it, one per group where nothing is cut."""
import pytest

import paper_2502_02175_amd as V
from test_gpu_attend import Cache, compare, i32, queries
from test_gpu_attend import DEV
from test_gpu_attend_tables import long_tables  # noqa: F401

pytestmark = pytest.mark.gpu


def items(p, seqs, pos, group, hq):
    import torch
    ws = torch.empty(V.vlac_attend_workspace_bytes(p, len(seqs), 1, hq), dtype=torch.uint8, device=DEV)
    V.vlac_attend_plan(p, i32(seqs), i32(pos), len(seqs), 1, hq, i32(group), ws)
    return int(ws[:4].view(torch.int32)[0])


@pytest.mark.parametrize("each,skip", [(1, None), (2, None), (2, 0), (3, 0), (3, 1)])
def test_many_groups_of_one_block_are_not_cut(long_tables, each, skip):  # noqa: F811
    """200 groups of a block each over 63 pages: 200 of 256 CUs for as long as the longest list.  skip: an entry of every group that
    is ignored (the first says nothing about the group's length)."""
    c = Cache(1, 64, 1, seed=each)
    base = [c._new(32) for _ in range(63)]
    at = 63 * 32 + 5
    s = [c.sequence(at + 1 + k, base) for k in range(each)]
    seqs, pos, group = [], [], []
    for g in range(200):
        seqs += s
        pos += [-1 if k == skip else at + k for k in range(each)]
        group += [g] * each
    p = c.pool()
    assert items(p, seqs, pos, group, 8) == 200
    compare(c, p, seqs, pos, queries(c, len(seqs), 1, 8), group)


def test_one_longer_list_among_many(long_tables):  # noqa: F811
    """(of 125 pages beside 199 of 100: the others last nearly as long)"""
    c = Cache(1, 64, 1, seed=4)
    base = [c._new(32) for _ in range(125)]
    long, short = c.sequence(125 * 32 + 1, base), c.sequence(100 * 32 + 1, base[:100])
    seqs, pos = [short] * 199 + [long], [100 * 32] * 199 + [125 * 32]
    p = c.pool()
    assert items(p, seqs, pos, list(range(200)), 8) == 200
    compare(c, p, seqs, pos, queries(c, 200, 1, 8), list(range(200)))


def test_few_long_lists_are_cut(long_tables):  # noqa: F811
    c = Cache(1, 64, 1, seed=5)
    s = c.sequence(130 * 32 + 1)
    p = c.pool()
    for n in (1, 20):
        assert items(p, [s] * n, [130 * 32] * n, list(range(n)), 8) > n
        compare(c, p, [s] * n, [130 * 32] * n, queries(c, n, 1, 8), list(range(n)))
