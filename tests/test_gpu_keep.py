"""Accepted paths of drafted trees, and the pages that keep them, against the plain model: every whole number and every value."""
import random

import pytest

import drafts_model as M
import paper_2502_02175_amd as V
from pages_model import E_RANGE, OK, PAGE, Pool, k_tile_at, pages_of, v_tile_at

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def i32(x):
    import torch
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def accept(parents, drafted, chosen):
    import torch
    n, T = len(parents), len(parents[0])
    path, count, token = torch.full((n, T), -9, dtype=torch.int32, device=DEV), i32([-9] * n), i32([-9] * n)
    V.vlac_tree_accept(i32(parents), i32(drafted), i32(chosen), n, T, path, count, token)
    return path.tolist(), count.tolist(), token.tolist()


@pytest.mark.parametrize("T", [1, 2, 7, 32, 255, 256, 257, 512])
@pytest.mark.parametrize("kind", ["random", "chain", "star", "holes", "roots"])
@pytest.mark.parametrize("tokens", [1, 2, 50])
def test_accept(T, kind, tokens):
    rng = random.Random(T * 31 + tokens)
    parents = [M.tree(rng, T, kind, rng.randint(1, T)) for _ in range(9)]
    if T > 4:
        parents[3][2], parents[4][3] = 2, 77777                 # (follows itself, follows nobody)
        parents[5][0] = -2
    drafted, chosen = ([[rng.randrange(tokens) for _ in range(T)] for _ in range(9)] for _ in range(2))
    path, count, token = accept(parents, drafted, chosen)
    for i in range(9):
        want, after = M.accept(parents[i], drafted[i], chosen[i])
        assert path[i] == want + [-1] * (T - len(want)) and count[i] == len(want) and token[i] == after


def test_accept_stops_where_nothing_may_follow():
    path, count, token = accept([[-1, 0, 1, 2], [-1, 0, 0, 2]], [[9, -1, 5, 6], [9, 3, 3, 4]], [[-1, 5, 6, 7], [3, -1, 4, -1]])
    assert path == [[0, -1, -1, -1], [0, 1, -1, -1]] and count == [1, 2] and token == [-1, -1]


class Both:
    """A pool on the GPU and its model, with random values everywhere."""

    def __init__(self, layers, hkv, hd, operand, n_pages, max_seqs, max_pages, seed=0):
        import torch
        self.hkv, self.hd = hkv, hd
        self.gpu, self.model = V.new_pages(layers, hkv, hd, operand, n_pages, max_seqs, max_pages, DEV), Pool(n_pages, max_seqs, max_pages)
        g = torch.Generator(device=DEV)
        g.manual_seed(seed)
        self.data = self.gpu.tensors[0].view(torch.int16).view(n_pages, layers, 2, hkv, PAGE * hd)
        self.data.copy_(torch.randint(-2 ** 15, 2 ** 15, self.data.shape, generator=g, device=DEV))

    def extend(self, seqs, tokens):
        pos = i32([0] * len(seqs))
        V.vlac_pages_extend(self.gpu, i32(seqs), len(seqs), tokens, pos)
        assert pos.tolist() == self.model.extend(seqs, tokens)
        return pos.tolist()

    def keep(self, seqs, pos, tokens, path, count):
        import torch
        want = self.data.clone()
        rows = [list(r) for r in self.model.table]
        for i, a, b in M.keep(self.model, seqs, pos, tokens, path, count):
            (pa, ra), (pb, rb) = divmod(a, PAGE), divmod(b, PAGE)
            for w, f in ((0, k_tile_at), (1, v_tile_at)):
                at = torch.tensor(f(self.hd), device=DEV)
                want[rows[seqs[i]][pb], :, w][..., at[rb]] = want[rows[seqs[i]][pa], :, w][..., at[ra]]
        full = [list(x) + [-1] * (tokens - len(x)) for x in path]
        V.vlac_pages_keep(self.gpu, i32(seqs), i32(pos), len(seqs), tokens, i32(full), i32(count))
        assert torch.equal(self.data, want)
        self.books()

    def books(self):
        _, refs, table, length, scratch = self.gpu.tensors
        assert refs.tolist() == self.model.refs and table.tolist() == self.model.table and length.tolist() == self.model.len
        assert V.vlac_pages_check(self.gpu, check=False) == self.model.check()
        assert not bool(scratch[16 + 3 * refs.numel():].any())   # the marks of sequences


@pytest.mark.parametrize("layers,hkv,hd,operand", [(1, 1, 64, 1), (3, 4, 64, 0), (2, 5, 128, 1), (1, 9, 128, 0)])
@pytest.mark.parametrize("tokens", [1, 2, 7, 33, 130, 512])
def test_keep(layers, hkv, hd, operand, tokens):
    rng = random.Random(tokens + hd)
    starts = [0, 1, 30, 31, 32, 33, 64, 100]
    b = Both(layers, hkv, hd, operand, sum(pages_of(x + tokens) for x in starts) * 2 + 20, 10, pages_of(100 + 3 * tokens) + 1, seed=tokens)
    seqs = list(range(8))
    for s, x in zip(seqs, starts):
        if x:
            b.extend([s], x)
    order = rng.sample(seqs, 8)
    for turn in range(3):
        pos = b.extend(order, tokens)
        path = [sorted(rng.sample(range(tokens), rng.randint(0, min(tokens, 20 if turn else tokens)))) for _ in order]
        path[0], path[1] = list(range(tokens)) if turn == 0 else [], [tokens - 1]
        if turn == 2:
            pos[2] = -1                                          # (skipped; its positions stay)
        b.keep(order, pos, tokens, path, [len(x) for x in path])
        if turn == 2:
            assert b.model.len[order[2]] > 0


def test_entries_that_do_not_fit():
    b = Both(2, 2, 64, 1, 60, 12, 6)
    T = 40
    b.extend([0, 1, 2, 3, 4, 5, 6, 7], 20)
    pos = b.extend([0, 1, 2, 3, 4, 5, 6, 7], T)
    good = list(range(1, 6))
    b.keep([0, 0, 99, -1, 1, 2, 3, 4, 5], pos[:1] * 4 + [19, 20, 20, 20, 20], T,
           [good, [3], good, good, good, [3, 3], [5, 4], [2, T], [0, 1, 2]], [5, 1, 5, 5, 5, 2, 2, 2, T + 1])
    b.keep([6, 7], [20, 20], T, [good, good], [-1, 5])
    assert b.model.len[0] == 25 and b.model.len[7] == 25 and b.model.len[5] == 20 + T
    # rows that would move into pages that another sequence holds; a path that moves nothing may end in one
    src, dst = i32([1, 2]), i32([10, 11])
    V.vlac_pages_fork(b.gpu, src, dst, 2)
    b.model.fork([1, 2], [10, 11])
    b.model.data = list(range(60))
    b.keep([1, 10, 2, 11], [20] * 4, T, [[0, 2], [0, 30], [0, 1, 2], []], [2, 2, 3, 0])
    # a length out of range, a table entry that names no page
    _, refs, table, length, _ = b.gpu.tensors
    length[3], b.model.len[3] = 7000, 7000
    row = table[4].tolist()
    table[4, 0] = 1 << 20
    before = b.data.clone()
    V.vlac_pages_keep(b.gpu, i32([3, 4]), i32([20, 20]), 2, T, i32([good + [-1] * (T - 5)] * 2), i32([5, 5]))
    assert V.vlac_pages_check(b.gpu, check=False) == E_RANGE and bool((b.data == before).all())
    assert length[3].item() == 7000 and length[4].item() == 20 + T and table[4].tolist()[1:] == row[1:]
    V.vlac_pages_keep(b.gpu, i32([]), i32([]), 0, T, i32([]), i32([]))
    assert V.vlac_pages_check(b.gpu, check=False) == OK


def test_many_entries():
    rng = random.Random(1)
    n, T = 1500, 3
    b = Both(1, 1, 64, 1, 2 * n + 8, n, 2)
    seqs = list(range(n))
    for first in range(0, n, 500):
        b.extend(seqs[first:first + 500], 30 + first // 500)
    pos = b.extend(seqs, T)
    path = [sorted(rng.sample(range(T), rng.randint(0, T))) for _ in seqs]
    b.keep(seqs, pos, T, path, [len(x) for x in path])


def test_more_work_than_workgroups():
    """4096 entries of 18 layers: a workgroup takes one after another, some of which do not fit for one row of theirs."""
    rng = random.Random(2)
    n, T, layers = 4096, 3, 18
    b = Both(layers, 1, 64, 1, 2 * n + 8, n, 2)
    seqs = list(range(n))
    b.extend(seqs, 30)
    pos = b.extend(seqs, T)
    path = [rng.choice([[2], [0, 2], [1, 2], [1], [2, 1], [0, 3], [1, 1], [], [0, 1, 2]]) for _ in seqs]
    b.keep(seqs, pos, T, path, [len(x) for x in path])


def test_offsets_beyond_32_bits():
    import torch
    layers, hkv, hd = 32, 32, 128
    n_pages = (1 << 32) // (layers * 2 * hkv * PAGE * hd) + 3
    p = V.new_pages(layers, hkv, hd, 1, n_pages, 1, 2, DEV)
    data, refs, table, length, _ = p.tensors
    table[0, 0], table[0, 1], length[0], refs[n_pages - 1], refs[0] = n_pages - 1, 0, 40, 1, 1
    d = data.view(torch.int16).view(n_pages, layers, 2, hkv, PAGE * hd)
    for pg in (0, n_pages - 1):
        d[pg] = torch.randint(-2 ** 15, 2 ** 15, d[pg].shape, device=DEV)
    want = {pg: d[pg].clone() for pg in (0, n_pages - 1)}
    for w, f in ((0, k_tile_at), (1, v_tile_at)):
        at = torch.tensor(f(hd), device=DEV)
        want[n_pages - 1][:, w][..., at[30]] = want[0][:, w][..., at[3]]
    V.vlac_pages_keep(p, i32([0]), i32([30]), 1, 10, i32([[5] + [-1] * 9]), i32([1]))
    assert V.vlac_pages_check(p, check=False) == OK and length[0].item() == 31 and refs[0].item() == 0
    for pg in want:
        assert torch.equal(d[pg], want[pg])
