"""Attention of trees of drafted tokens over pages against its definition in 64 bits: trees of every shape and size, nodes that are not
there, NaN wherever nobody looks, shared prefixes, lists that are cut; a chain is what the attention of plain tokens makes of it, bit for bit."""
import math
import random

import pytest

import drafts_model as M
import paper_2502_02175_amd as V
from pages_model import E_RANGE, OK, PAGE, k_tile_at, pages_of, v_tile_at
from test_gpu_attend import LAYOUTS, Cache, i32, queries

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def seen_by(parents, pos):
    """[T, pos + T]: what each node sees."""
    import torch
    T = len(parents)
    see = torch.zeros((T, pos + T), dtype=torch.bool)
    for t in range(T):
        up = M.lineage(parents, t)
        if up is not None:
            see[t, :pos] = True
            see[t, [pos + u for u in up]] = True
    return see.to(DEV)


def definition(cache, seqs, pos, q, trees, layer=0):
    """-> out, and how far rounding may take each value: weights and result are rounded to the type (half a step each), scores are sums
    of hd products in fp32, relative to the sum of the products' sizes, sums of weights in fp32."""
    import torch
    n, T, hq, hd = q.shape
    out = torch.zeros(q.shape, dtype=torch.float64, device=DEV)
    tol = torch.full_like(out, 2.0 ** -25)
    half = torch.finfo(cache.dt).eps / 2
    for i, (s, p) in enumerate(zip(seqs, pos)):
        if p < 0:
            continue
        see = seen_by(trees[i], p)
        there = see.any(1)
        k, v = (x[:p + T].permute(1, 0, 2).repeat_interleave(hq // cache.hkv, 0) for x in cache.kv(s, layer))
        used = see.any(0)
        k, v = k * 1.0, v * 1.0
        k[:, ~used] = 0.0
        v[:, ~used] = 0.0
        qq = q[i].double().permute(1, 0, 2)
        qq = torch.where(there[None, :, None], qq, 0.0)
        sc = qq @ k.transpose(1, 2) / math.sqrt(hd)
        size = (qq.abs() @ k.abs().transpose(1, 2) / math.sqrt(hd)).masked_fill(~see, 0).amax()
        w = torch.nan_to_num(torch.softmax(sc.masked_fill(~see, -math.inf), 2))
        y, spread = ((w @ x).permute(1, 0, 2) for x in (v, v.abs()))
        fp32 = 2.0 ** -23 * (2 * (hd + 2) * size + 2 * (p + T) + 16)
        out[i], tol[i] = y, half * y.abs() + (half + fp32) * spread + 2.0 ** -25
    return out, tol


def run(p, cache, seqs, pos, q, trees, group=None, layer=0, places=True):
    import torch
    n, T, hq, hd = q.shape
    ws = torch.empty(V.vlac_attend_tree_workspace_bytes(p, n, T, hq), dtype=torch.uint8, device=DEV)
    ws.fill_(0xFF)
    out = torch.full((n, T, hq, hd), 7.0, dtype=cache.dt, device=DEV)
    where = torch.full((n, T), -9, dtype=torch.int32, device=DEV) if places else None
    V.vlac_attend_tree_plan(p, i32(seqs), i32(pos), n, T, hq, None if group is None else i32(group), i32(trees), where, ws)
    V.vlac_attend_tree(p, layer, n, T, hq, q, out, ws)
    return out, where


def compare(cache, p, seqs, pos, q, trees, group=None, layer=0):
    import torch
    got, where = run(p, cache, seqs, pos, q, trees, group, layer)
    want, tol = definition(cache, seqs, pos, q, trees, layer)
    assert bool(torch.isfinite(got).all())
    err = (got.double() - want).abs()
    assert bool((err <= tol).all()), "%.3g over the bound" % float((err / tol).max())
    for i, t in enumerate(trees):
        assert where[i].tolist() == ([-1] * len(t) if pos[i] < 0 else M.places(t, pos[i]))
        for k in range(len(t)):
            if M.lineage(t, k) is None:
                assert not bool(got[i, k].any())
    return got


def spoil(cache, seqs, pos, trees):
    """NaN in the slots of nodes that are not there (the cache's pages, before the pool is made)."""
    for s, p, t in zip(seqs, pos, trees):
        for k in range(len(t)):
            if p >= 0 and M.lineage(t, k) is None:
                cache.pages[cache.seqs[s][0][(p + k) // PAGE]][:, :, (p + k) % PAGE] = float("nan")


@pytest.mark.parametrize("hq,hkv,hd", LAYOUTS)
@pytest.mark.parametrize("operand", [0, 1])
@pytest.mark.parametrize("T", [1, 5, 40])
def test_groups_of_several_prefixes(hq, hkv, hd, operand, T):
    c = Cache(hkv, hd, operand, seed=hq + hd + T)
    seqs, pos, group, trees = [], [], [], []
    rng = random.Random(T + hq)
    kinds = ["random", "chain", "star", "holes", "roots"]
    for g, stem in enumerate((75, 64, 1, 31, 200)):
        base = [c._new(PAGE) for _ in range(stem // PAGE)]
        for k in range(1 + g % 3 * 2):
            own = (7 * k + 3 * g) % 45
            seqs.append(c.sequence(stem + own + T, base))
            pos.append(stem + own)
            group.append(g * 3 - 2)
            trees.append(M.tree(rng, T, kinds[(g + k) % 5], rng.randint(1, T)))
    spoil(c, seqs, pos, trees)
    q = queries(c, len(seqs), T, hq)
    p = c.pool()
    got = compare(c, p, seqs, pos, q, trees, group)
    compare(c, p, seqs, pos, q, trees, None)                    # one group that shares nothing
    again, _ = run(p, c, seqs, pos, q, trees, group, places=False)
    assert bool((got == again).all())                           # the same bits whenever it runs
    assert V.vlac_pages_check(p, check=False) == OK


@pytest.mark.parametrize("pos", [0, 1, 30, 31, 32, 33, 63, 500, 2500])
@pytest.mark.parametrize("T", [1, 2, 31, 32, 33, 64, 65, 200, 512])
def test_one_tree_of_any_size(pos, T):
    hq, hkv, hd, operand = (12, 2, 128, 0) if T % 2 else (4, 4, 64, 1)
    c = Cache(hkv, hd, operand, seed=pos + T)
    s = c.sequence(pos + T)
    rng = random.Random(pos * 1000 + T)
    p = None
    for kind in ("random", "chain", "holes"):
        t = M.tree(rng, T, kind)
        if p is None:
            p = c.pool()
        compare(c, p, [s], [pos], queries(c, 1, T, hq), [t])


@pytest.mark.parametrize("n,T,hq,hkv,hd,stem,operand", [
    (2, 7, 4, 4, 64, 64 * 70, 1),       # few columns over a long stem: many parts
    (8, 16, 32, 32, 128, 1057, 1),      # several column blocks of several entries
    (40, 1, 32, 32, 128, 64 * 33, 1),
    (33, 3, 8, 2, 64, 700, 1),
    (3, 100, 6, 2, 128, 77, 0),
    (2, 64, 8, 1, 128, 5000, 0),        # parts, with masks that span them
    (1200, 2, 4, 2, 64, 40, 1)])        # more entries than the planning workgroup has threads
def test_columns_and_parts(n, T, hq, hkv, hd, stem, operand):
    c = Cache(hkv, hd, operand, seed=n)
    base = [c._new(PAGE) for _ in range(stem // PAGE)]
    pos = [stem + (3 * i) % 7 for i in range(n)]
    seqs = [c.sequence(pos[i] + T, base) for i in range(n)]
    rng = random.Random(n)
    trees = [M.tree(rng, T, "holes" if i % 3 == 2 else "random", T - i % T) for i in range(n)]
    spoil(c, seqs, pos, trees)
    compare(c, c.pool(), seqs, pos, queries(c, n, T, hq), trees, None)


@pytest.mark.parametrize("n,T,hq,hkv,hd,stem,operand", [(4, 9, 4, 4, 64, 50, 1), (6, 40, 12, 2, 128, 300, 0), (2, 5, 32, 32, 128, 4000, 1)])
def test_a_chain_is_plain_text(n, T, hq, hkv, hd, stem, operand):
    import torch
    c = Cache(hkv, hd, operand, seed=T)
    base = [c._new(PAGE) for _ in range(stem // PAGE)]
    pos = [stem + 5 * i % 29 for i in range(n)]
    seqs = [c.sequence(pos[i] + T, base) for i in range(n)]
    p, q = c.pool(), queries(c, n, T, hq)
    got, _ = run(p, c, seqs, pos, q, [M.tree(None, T, "chain")] * n)
    ws = torch.empty(V.vlac_attend_workspace_bytes(p, n, T, hq), dtype=torch.uint8, device=DEV)
    want = torch.empty_like(got)
    V.vlac_attend_plan(p, i32(seqs), i32(pos), n, T, hq, None, ws)
    V.vlac_attend_shared(p, 0, n, T, hq, q, want, ws)
    assert torch.equal(got.view(torch.int16), want.view(torch.int16))


@pytest.mark.parametrize("hq,hkv,hd,operand,T,stem", [(4, 4, 64, 1, 6, 40), (12, 2, 128, 0, 30, 70), (2, 1, 64, 0, 9, 3000)])
@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf")])
def test_what_lies_at_a_node_that_is_not_seen(hq, hkv, hd, operand, T, stem, value):
    """K and V of node 2 hold it: only node 2 and those that follow it notice."""
    import torch
    c = Cache(hkv, hd, operand, seed=T)
    s = c.sequence(stem + T)
    rng = random.Random(T)
    tree = M.tree(rng, T, "random")
    hit = [t for t in range(T) if 2 in M.lineage(tree, t)]
    q = queries(c, 1, T, hq)
    clean, _ = run(c.pool(), c, [s], [stem], q, [tree])
    at = stem + 2
    page = c.pages[c.seqs[s][0][at // PAGE]]
    for which in (0, 1):                                        # K, then V
        kept = page[:, which, at % PAGE].clone()
        page[:, which, at % PAGE] = value
        got, _ = run(c.pool(), c, [s], [stem], q, [tree])
        page[:, which, at % PAGE] = kept
        others = [t for t in range(T) if t not in hit]
        assert bool(torch.isfinite(got[0, others]).all())
        # (a value nobody sees may move a sum's order, never its value by more than rounding: twice the bound of either)
        _, tol = definition(c, [s], [stem], q, [tree])
        assert bool(((got[0, others].double() - clean[0, others].double()).abs() <= 2 * tol[0, others]).all())
        if which == 1:
            bad = got[0, hit]
            assert bool(torch.isnan(bad).all() if math.isnan(value) else torch.isinf(bad).all())
        elif math.isnan(value):
            assert bool(torch.isnan(got[0, hit]).all())


def test_entries_and_parents_that_do_not_fit():
    import torch
    c = Cache(2, 64, 1, seed=9)
    T = 6
    pos = [40, -1, 12, 70, 33]
    seqs = [c.sequence(x + T) for x in (40, 50, 12, 70, 33)]
    trees = [[-1, 0, 0, 1, 2, 3], [-1] * 6, [-1, 0, 1, 2, 3, 4], [-1, 5, 0, -3, 3, 2], [0, -1, 1, 1, 2, 2]]
    p, q = c.pool(), queries(c, 5, T, 4)
    compare(c, p, seqs, pos, q, trees)                          # (a parent that is no earlier node: there is no such node)
    assert V.vlac_pages_check(p, check=False) == E_RANGE and V.vlac_pages_check(p, check=False) == OK
    # an unknown sequence, one that is too short, a negative position: rows of zeros, places -1
    got, where = run(p, c, [seqs[0], 99, seqs[2]], [41, 3, -5], q[:3], [trees[0]] * 3)
    assert not bool(got.any()) and bool((where == -1).all())
    assert V.vlac_pages_check(p, check=False) == E_RANGE
    out = torch.full_like(q, 7.0)
    # a workspace of the other kind of plan is not used
    for tree_first in (True, False):
        ws = torch.zeros(V.vlac_attend_tree_workspace_bytes(p, 5, T, 4), dtype=torch.uint8, device=DEV)
        if tree_first:
            V.vlac_attend_tree_plan(p, i32(seqs), i32(pos), 5, T, 4, None, i32(trees), None, ws)
            V.vlac_pages_check(p, check=False)
            V.vlac_attend_shared(p, 0, 5, T, 4, q, out, ws)
        else:
            V.vlac_attend_plan(p, i32(seqs), i32(pos), 5, T, 4, None, ws)
            V.vlac_attend_tree(p, 0, 5, T, 4, q, out, ws)
        assert V.vlac_pages_check(p, check=False) == E_RANGE and bool((out == 7).all())
    V.vlac_attend_tree(p, 0, 0, T, 4, None, None, None)


def test_layers_and_strided_queries():
    import torch
    c = Cache(2, 128, 1, seed=4, layers=3)
    T, hq = 11, 6
    pos = [100, 37]
    seqs = [c.sequence(x + T) for x in pos]
    trees = [M.some_tree(1, T), M.some_tree(2, T, "holes")]
    p = c.pool()
    joint = queries(c, 2, T, hq + 4)
    ws = torch.empty(V.vlac_attend_tree_workspace_bytes(p, 2, T, hq), dtype=torch.uint8, device=DEV)
    V.vlac_attend_tree_plan(p, i32(seqs), i32(pos), 2, T, hq, None, i32(trees), None, ws)
    for layer in (2, 0, 1):
        q = joint[:, :, :hq]
        out = torch.empty((2, T, hq, 128), dtype=c.dt, device=DEV)
        V.vlac_attend_tree(p, layer, 2, T, hq, q, out, ws)
        want, tol = definition(c, seqs, pos, q, trees, layer)
        assert bool(((out.double() - want).abs() <= tol).all())


def test_one_sequence_in_several_entries():
    """Different trees over the same slots of one sequence, and the same entry twice."""
    for hq, hkv, hd, T, stem in ((4, 4, 64, 12, 50), (12, 2, 128, 30, 2300)):
        c = Cache(hkv, hd, 1, seed=T)
        s, other = c.sequence(stem + T), c.sequence(9 + T)
        trees = [M.some_tree(k, T, kind) for k, kind in enumerate(("random", "chain", "random", "roots"))]
        seqs, pos = [s, s, other, s], [stem, stem, 9, stem]
        p, q = c.pool(), queries(c, 4, T, hq)
        for group in (None, [1, 1, 2, 2], [0, 1, 2, 3]):
            compare(c, p, seqs, pos, q, trees, group)
        q[1] = q[0]                                             # (the order of the sums is each entry's own)
        compare(c, p, [s, s], [stem, stem], q[:2], [trees[0]] * 2)


def test_two_workspaces_on_two_streams():
    import torch
    c = Cache(4, 128, 0, seed=2)
    T, hq = 20, 8
    pos = [300, 40, 2200]
    seqs = [c.sequence(x + T) for x in pos]
    trees = [[M.some_tree(10 * k + i, T) for i in range(3)] for k in range(2)]
    p = c.pool()
    q = [queries(c, 3, T, hq) for _ in range(2)]
    want = [run(p, c, seqs, pos, q[k], trees[k])[0] for k in range(2)]
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in range(2)], [None, None]
    for _ in range(5):
        for k in range(2):
            with torch.cuda.stream(streams[k]):
                got[k] = run(p, c, seqs, pos, q[k], trees[k])[0]
        torch.cuda.synchronize()
        assert all(torch.equal(a.view(torch.int16), b.view(torch.int16)) for a, b in zip(want, got))
