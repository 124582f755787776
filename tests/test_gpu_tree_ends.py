"""Attention of trees at the ends of what is allowed: the longest list, the most nodes and rows, the most heads, the longest sequence, offsets
beyond 32 bits."""
import random

import pytest

import drafts_model as M
import paper_2502_02175_amd as V
from pages_model import OK, PAGE
from test_gpu_attend import Cache, i32, queries
from test_gpu_tree import compare, definition, run

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def check_some(c, p, seqs, pos, q, trees, group, some):
    """All entries in one call, the listed ones looked at."""
    got, where = run(p, c, seqs, pos, q, trees, group)
    want, tol = definition(c, [seqs[i] for i in some], [pos[i] for i in some], q[some], [trees[i] for i in some])
    assert bool(((got[some].double() - want).abs() <= tol).all())
    for i in some:
        assert where[i].tolist() == M.places(trees[i], pos[i])
    assert V.vlac_pages_check(p, check=False) == OK


def test_the_longest_list():
    """4096 entries in groups of one, two, three, ... of them."""
    n, T = 4096, 5
    c = Cache(2, 64, 1, seed=2)
    stems = [[c._new(PAGE)] for _ in range(100)]
    group, g = [], 0
    while len(group) < n:
        group += [g] * min(g + 1, n - len(group))
        g += 1
    pos = [32 + (7 * i) % 31 for i in range(n)]
    seqs = [c.sequence(pos[i] + T, stems[group[i]]) for i in range(n)]
    trees = [M.some_tree(i % 40, T, ("random", "holes", "chain", "roots")[i % 4]) for i in range(n)]
    check_some(c, c.pool(), seqs, pos, queries(c, n, T, 4), trees, group, list(range(0, n, 61)) + [n - 1])


@pytest.mark.parametrize("hq,hkv,hd,operand", [(1, 1, 64, 1), (2, 1, 128, 0)])
def test_a_million_nodes(hq, hkv, hd, operand):
    """2048 trees of 512 places."""
    n, T = 2048, 512
    c = Cache(hkv, hd, operand, seed=hq)
    pos = [(5 * i) % 37 for i in range(n)]
    base = [c._new(PAGE) for _ in range(34)]
    own = [c.sequence(x + T) if i % 128 == 0 else None for i, x in enumerate(pos)]
    seqs = [s if s is not None else c.sequence(pos[i] + T, random.Random(i).sample(base, 17)) for i, s in enumerate(own)]
    trees = [M.some_tree(i % 16, T, ("random", "holes", "chain", "roots")[i % 4]) for i in range(n)]
    check_some(c, c.pool(), seqs, pos, queries(c, n, T, hq), trees, list(range(n)), list(range(0, n, 157)) + [n - 1])


@pytest.mark.parametrize("hq,hkv,hd,operand,n,T", [(1024, 1, 64, 1, 3, 2), (1024, 1024, 64, 0, 2, 3), (1024, 8, 128, 1, 2, 3),
                                                   (1000, 125, 64, 1, 3, 2), (1023, 3, 128, 0, 1, 2)])
@pytest.mark.parametrize("columns", [0, 80])
def test_many_heads(hq, hkv, hd, operand, n, T, columns):
    c = Cache(hkv, hd, operand, seed=hq + hkv)
    base = [c._new(PAGE) for _ in range(2)]
    pos = [64 + 9 * i for i in range(n)]
    seqs = [c.sequence(x + T, base) for x in pos]
    if columns:                                                # (a table with room for long lists)
        c.sequence(PAGE * columns, base * (columns // 2))
    p = c.pool()
    compare(c, p, seqs, pos, queries(c, n, T, hq), [M.some_tree(i, T) for i in range(n)])
    assert V.vlac_pages_check(p, check=False) == OK


@pytest.mark.parametrize("hq,n,T", [(1, 1, 33), (4, 3, 6)])
def test_the_longest_sequence(monkeypatch, hq, n, T):
    """2^20 positions: 32768 pages, each of 1024 pages 32 times; the tree takes the last."""
    make = V.new_pages
    monkeypatch.setattr(V, "new_pages", lambda *a: make(*a[:6], min(a[6], 32768), a[7]))
    c = Cache(1, 64, 1, seed=n)
    base = [c._new(PAGE) for _ in range(1024)]
    length = 1 << 20
    seqs = [c.sequence(length, base * 31 + base[:1024 - i]) for i in range(n)]
    p = c.pool()
    trees = [M.some_tree(i, T) for i in range(n)]
    for group in (None, list(range(n))):
        compare(c, p, seqs, [length - T] * n, queries(c, n, T, hq), trees, group)
    assert V.vlac_pages_check(p, check=False) == OK


@pytest.mark.parametrize("hq", [32, 64])
def test_offsets_beyond_32_bits(hq):
    """A pool of 8.7 GB (more than 2^32 values), a sequence in its last pages."""
    import torch
    T, pos, layers, hkv, hd, n_pages = 9, 61, 32, 32, 128, 516
    c = Cache(hkv, hd, 1, seed=hq)
    s = c.sequence(pos + T)
    small = c.pool()
    p = V.new_pages(layers, hkv, hd, 1, n_pages, 2, 4, DEV)
    data, refs, table, length, _ = p.tensors
    here, there = (x.tensors[0].view(torch.int16).view(-1, k, 2 * hkv * PAGE * hd) for x, k in ((small, 1), (p, layers)))
    for j, pg in enumerate(small.tensors[2][s].tolist()):
        if pg >= 0:
            there[n_pages - 1 - j, layers - 1] = here[pg, 0]
            table[1, j], refs[n_pages - 1 - j] = n_pages - 1 - j, 1
    length[1] = pos + T
    q, trees = queries(c, 1, T, hq), [M.some_tree(3, T, "holes")]
    got, where = run(p, c, [1], [pos], q, trees, layer=layers - 1)
    want, tol = definition(c, [s], [pos], q, trees)
    assert bool(((got.double() - want).abs() <= tol).all()) and where[0].tolist() == M.places(trees[0], pos)
    assert V.vlac_pages_check(p, check=False) == OK
