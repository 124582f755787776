"""Attention over pages against its definition in 64 bits: every head layout, lengths from one position on, groups that share
much, little or nothing, rows that see nothing, NaN where no token was written."""
import math
import random

import pytest

import paper_2502_02175_amd as V
from pages_model import E_RANGE, OK, PAGE, k_tile_at, pages_of, v_tile_at

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def i32(x):
    import torch
    return torch.tensor(x, dtype=torch.int32, device=DEV)


class Cache:
    """A pool whose sequences are made on the host: `stem` positions of group g come first in each of its
    sequences (full pages shared, unless apart), the rest is its own."""

    def __init__(self, hkv, hd, operand, seed, layers=1):
        import torch
        self.hkv, self.hd, self.operand, self.layers = hkv, hd, operand, layers
        self.dt = torch.bfloat16 if operand == 0 else torch.float16
        self.g = torch.Generator(device=DEV)
        self.g.manual_seed(seed)
        self.pages, self.seqs = [], []                      # K and V [32, hkv, hd] of every page; (pages, length)

    def _new(self, filled, scale=1.0):
        import torch
        x = (scale * torch.randn((self.layers, 2, PAGE, self.hkv, self.hd), generator=self.g, device=DEV)).to(self.dt)
        x[:, :, filled:] = float("nan")
        self.pages.append(x)
        return len(self.pages) - 1

    def sequence(self, length, shared=()):
        mine = list(shared)
        while len(mine) < pages_of(length):
            mine.append(self._new(min(PAGE, length - PAGE * len(mine))))
        self.seqs.append((mine, length))
        return len(self.seqs) - 1

    def pool(self, extra_seqs=2, seed=0):
        import torch
        n = len(self.pages) + 5
        where = random.Random(seed).sample(range(n), n)     # pages lie anywhere
        p = V.new_pages(self.layers, self.hkv, self.hd, self.operand, n, len(self.seqs) + extra_seqs,
                        max([len(m) for m, _ in self.seqs] + [1]) + 1, DEV)
        data, refs, table, length, _ = p.tensors
        data.fill_(0xFF)
        d = data.view(torch.int16).view(n, self.layers, 2, self.hkv, PAGE * self.hd)
        ka, va = (torch.tensor(f(self.hd), device=DEV).flatten() for f in (k_tile_at, v_tile_at))
        if self.pages:
            x = torch.stack(self.pages).permute(0, 1, 2, 4, 3, 5).reshape(len(self.pages), self.layers, 2, self.hkv, -1).view(torch.int16)
            y = torch.empty_like(x)
            y[:, :, 0, :, ka] = x[:, :, 0]
            y[:, :, 1, :, va] = x[:, :, 1]
            d[torch.tensor(where[:len(self.pages)], device=DEV)] = y
        rows, count = [[-1] * table.shape[1] for _ in range(table.shape[0])], [0] * n
        for s, (mine, _) in enumerate(self.seqs):
            for j, pg in enumerate(mine):
                rows[s][j] = where[pg]
                count[where[pg]] += 1
        table.copy_(i32(rows))
        refs.copy_(i32(count))
        length.copy_(i32([l for _, l in self.seqs] + [0] * extra_seqs))
        return p

    def kv(self, s, layer=0):
        """K and V of sequence s in 64 bits, [length, hkv, hd]."""
        import torch
        mine, n = self.seqs[s]
        x = torch.cat([self.pages[pg][layer] for pg in mine], 1)[:, :n].double()
        return x[0], x[1]


def definition(cache, seqs, pos, q, layer=0):
    """-> out and, per value, how far rounding may take it: the weights are rounded to the type (half a step each), the result
    once more; scores are sums of hd products in fp32 and their exponentials carry that error and the chip's own."""
    import torch
    n, T, hq, hd = q.shape
    out = torch.zeros(q.shape, dtype=torch.float64, device=DEV)
    tol = torch.zeros_like(out)
    half = torch.finfo(cache.dt).eps / 2
    for i, (s, p) in enumerate(zip(seqs, pos)):
        if p < 0:
            continue
        k, v = (x[:p + T].permute(1, 0, 2).repeat_interleave(hq // cache.hkv, 0) for x in cache.kv(s, layer))
        qq = q[i].double().permute(1, 0, 2)
        sc = qq @ k.transpose(1, 2) / math.sqrt(hd)
        gone = torch.arange(p + T, device=DEV)[None, :] > p + torch.arange(T, device=DEV)[:, None]
        size = (qq.abs() @ k.abs().transpose(1, 2) / math.sqrt(hd)).masked_fill(gone, 0).amax()
        w = torch.softmax(sc.masked_fill(gone, -math.inf), 2)
        y = (w @ v).permute(1, 0, 2)
        spread = (w @ v.abs()).permute(1, 0, 2)
        # fp32: (hd + 2) roundings of a score, relative to the sum of its products' sizes; (p + T) of each sum, at most
        fp32 = 2.0 ** -23 * (2 * (hd + 2) * size + 2 * (p + T) + 16)
        out[i], tol[i] = y, half * y.abs() + (half + fp32) * spread + 2.0 ** -25
    return out, tol


def run(p, cache, seqs, pos, q, group=None, layer=0, out=None):
    import torch
    n, T, hq, hd = q.shape
    ws = torch.empty(V.vlac_attend_workspace_bytes(p, n, T, hq), dtype=torch.uint8, device=DEV)
    ws.fill_(0xFF)
    if out is None:
        out = torch.full((n, T, hq, hd), 7.0, dtype=cache.dt, device=DEV)
    V.vlac_attend_plan(p, i32(seqs), i32(pos), n, T, hq, None if group is None else i32(group), ws)
    V.vlac_attend_shared(p, layer, n, T, hq, q, out, ws)
    return out


def compare(cache, p, seqs, pos, q, group=None, layer=0):
    import torch
    got = run(p, cache, seqs, pos, q, group, layer)
    want, tol = definition(cache, seqs, pos, q, layer)
    err = (got.double() - want).abs()
    assert bool(torch.isfinite(got).all())
    assert bool((err <= tol).all()), "%.3g over the bound %.3g" % (float((err / tol).max()), 1.0)
    return got


def queries(cache, n, T, hq, scale=2.0):
    import torch
    return (scale * torch.randn((n, T, hq, cache.hd), generator=cache.g, device=DEV)).to(cache.dt)


LAYOUTS = [(4, 4, 64), (32, 32, 128), (12, 2, 128), (16, 4, 64), (8, 1, 128), (6, 3, 64), (64, 1, 64), (40, 1, 128), (1, 1, 64)]


@pytest.mark.parametrize("hq,hkv,hd", LAYOUTS)
@pytest.mark.parametrize("operand", [0, 1])
@pytest.mark.parametrize("T", [1, 5])
def test_groups_of_several_prefixes(hq, hkv, hd, operand, T):
    c = Cache(hkv, hd, operand, seed=hq + hd + T)
    seqs, pos, group = [], [], []
    for g, stem in enumerate((75, 64, 1, 31, 200)):
        base = [c._new(PAGE) for _ in range(stem // PAGE)]
        for k in range(1 + g % 3 * 2):
            own = (7 * k + 3 * g) % 45
            s = c.sequence(stem + own + T, base)
            seqs.append(s)
            pos.append(stem + own)
            group.append(g * 3 - 2)
    q = queries(c, len(seqs), T, hq)
    p = c.pool()
    got = compare(c, p, seqs, pos, q, group)
    compare(c, p, seqs, pos, q, None)                          # one group that shares nothing
    again = run(p, c, seqs, pos, q, group)
    assert bool((got == again).all())                          # the same bits whenever it runs
    assert V.vlac_pages_check(p, check=False) == OK


@pytest.mark.parametrize("length", [1, 2, 31, 32, 33, 63, 64, 65, 129, 1000, 2049])
@pytest.mark.parametrize("hq,hkv,hd,operand", [(4, 4, 64, 1), (12, 2, 128, 0)])
def test_one_sequence_of_any_length(length, hq, hkv, hd, operand):
    c = Cache(hkv, hd, operand, seed=length)
    for T in (1, min(length, 3), min(length, 40), length if length < 300 else 1):
        s = c.sequence(length)
        p = c.pool()
        compare(c, p, [s], [length - T], queries(c, 1, T, hq))


@pytest.mark.parametrize("n,T,hq,hkv,hd,stem,operand", [
    (2, 1, 4, 4, 64, 64 * 70, 1),       # few columns over a long stem: many parts
    (40, 1, 32, 32, 128, 64 * 33, 1),   # two column blocks
    (100, 1, 2, 2, 128, 1500, 0),      # four column blocks
    (33, 3, 8, 2, 64, 700, 1),        # thirteen column blocks, the last of one column... of 396 columns
    (16, 64, 32, 32, 64, 2304, 1),     # a wave's own column block over 72 pages, no parts
    (3, 100, 6, 2, 128, 77, 0),         # tokens that fill several blocks of their own
    (1200, 1, 4, 2, 64, 40, 1)])        # more entries than the planning workgroup has threads
def test_columns_and_parts(n, T, hq, hkv, hd, stem, operand):
    c = Cache(hkv, hd, operand, seed=n)
    base = [c._new(PAGE) for _ in range(stem // PAGE)]
    pos = [stem + (3 * i) % 7 for i in range(n)]
    seqs = [c.sequence(pos[i] + T, base) for i in range(n)]
    compare(c, c.pool(), seqs, pos, queries(c, n, T, hq), None)


def test_own_parts_behind_a_short_stem():
    """Own segments of very different lengths, one of them long enough for parts."""
    c = Cache(2, 128, 1, seed=3)
    base = [c._new(PAGE)]
    pos = [32, 33, 500, 40, 3000, 64]
    seqs = [c.sequence(x + 1, base) for x in pos]
    compare(c, c.pool(), seqs, pos, queries(c, 6, 1, 8), [0] * 6)


def test_groups_are_a_hint():
    """Labels that join sequences of other stems, split those of one stem, or come in no order."""
    c = Cache(2, 64, 1, seed=4)
    stems = [[c._new(PAGE) for _ in range(4)] for _ in range(2)]
    pos = [130, 135, 140, 128, 150, 129]
    seqs = [c.sequence(x + 1, stems[i % 2]) for i, x in enumerate(pos)]
    p = c.pool()
    q = queries(c, 6, 1, 4)
    for group in (None, [0] * 6, [0, 1, 0, 1, 0, 1], [5, 5, 5, -5, -5, -5], list(range(6))):
        compare(c, p, seqs, pos, q, group)
    compare(c, p, [seqs[0]] * 3 + [seqs[1]] * 3, [130, 100, 7, 135, 0, 31], q, [0, 0, 0, 1, 1, 1])   # one sequence, several positions
    half = c.sequence(110, stems[0][:2])                      # stems that part inside
    p = c.pool()
    compare(c, p, [seqs[0], half, seqs[2], seqs[4], half, half], [130, 109, 140, 150, 70, 64], q, [0] * 6)


def test_entries_that_do_not_fit_get_zeros():
    import torch
    c = Cache(2, 64, 0, seed=5)
    base = [c._new(PAGE) for _ in range(2)]
    good = [c.sequence(70 + i, base) for i in range(3)]
    p = c.pool()
    empty = len(c.seqs)
    seqs = [good[0], 99, good[1], -1, empty, good[2], good[2], good[0]]
    pos = [60, 3, -1, 0, 0, 71, 2 ** 31 - 1, -5]             # 71 + 2 tokens: one behind the end
    q = queries(c, 8, 2, 4)
    out = run(p, c, seqs, pos, q, [0] * 8)
    assert V.vlac_pages_check(p, check=False) == E_RANGE
    want, tol = definition(c, seqs[:1], pos[:1], q[:1])
    assert bool(((out[:1].double() - want).abs() <= tol).all())
    assert not bool(out[1:].any())
    out = run(p, c, seqs[1:5], pos[1:5], q[1:5], None)        # nobody left in the group
    assert not bool(out.any())
    V.vlac_pages_check(p, check=False)
    out = run(p, c, [good[1]] * 2, [-1, -1], q[:2], None)     # skipped, and no error
    assert not bool(out.any()) and V.vlac_pages_check(p, check=False) == OK
    assert run(p, c, [], [], q[:0]).numel() == 0


@pytest.mark.parametrize("operand", [0, 1])
def test_values_at_the_ends_of_the_type(operand):
    import torch
    c = Cache(2, 64, operand, seed=6)
    s = c.sequence(100)
    big = torch.finfo(c.dt).max
    # scores far apart (one position takes all), huge values of V, and equal scores of the lowest value
    c.pages[0][:, 0, 5] = 60.0
    c.pages[1][:, 1, 3] = big
    c.pages[2][:, 1, 0] = -big
    p = c.pool()
    q = queries(c, 1, 1, 4, 8.0)
    got, (want, tol) = run(p, c, [s], [99], q), definition(c, [s], [99], q)
    assert bool(((got.double() - want).abs() <= tol).all())
    q = torch.full((1, 1, 4, 64), -big, dtype=c.dt, device=DEV)
    c.pages[0][:, 0] = 1.0
    for pg in c.pages[1:]:
        pg[:, 0] = 1.0
    p = c.pool()
    got, (want, _) = run(p, c, [s], [99], q), definition(c, [s], [99], q)    # all scores -big * 8, equal
    if 64 * big / 8 > torch.finfo(torch.float32).max:
        # bf16: a score is 64 products of -3.39e38, its sum -2.2e40, and fp32 (in which the scores are defined) ends at
        # 3.40e38: every score is minus infinity, and the softmax of nothing but those is no number
        assert bool(torch.isnan(got).all())
        return
    half = torch.finfo(c.dt).eps / 2
    spread = torch.cat([pg[0, 1] for pg in c.pages], 0)[:100].double().abs().mean(0).repeat_interleave(2, 0)
    assert bool(((got.double() - want).abs()[0, 0] <= (4 * half + 1e-5) * spread).all())


def test_nan_and_infinity_stay_where_they_are_seen():
    import torch
    c = Cache(2, 64, 1, seed=7)
    base = [c._new(PAGE) for _ in range(2)]
    a, b = c.sequence(80, base), c.sequence(90, base)
    d = c.sequence(80, base)
    own = c.seqs[d][0][2]
    c.pages[own][:, 1, 10, 0, 3] = float("inf")              # V of position 74, kv head 0, feature 3
    c.pages[own][:, 0, 12, 1, 0] = float("nan")              # K of position 76, kv head 1
    p = c.pool()
    q = queries(c, 3, 4, 4)
    pos = [70, 80, 73]
    out = run(p, c, [a, b, d], pos, q, [0, 0, 0])
    want, tol = definition(c, [a, b], pos[:2], q[:2])
    assert bool(((out[:2].double() - want).abs() <= tol).all())
    assert bool(torch.isfinite(out[2, 0]).all())                # position 73 sees neither
    assert bool(torch.isinf(out[2, 1:, :2, 3]).all()) and bool(torch.isfinite(out[2, 1:3, :2, 4:]).all())
    assert bool(torch.isfinite(out[2, :3, 2:]).all()) and bool(torch.isnan(out[2, 3, 2:]).all())


def test_layers_strided_queries_and_what_lies_around():
    """A layer in the middle, queries as columns of a joint projection, nothing written outside out and workspace."""
    import torch
    c = Cache(2, 128, 0, seed=8, layers=3)
    base = [c._new(PAGE) for _ in range(3)]
    pos = [96, 99, 120, 140]
    seqs = [c.sequence(x + 2, base) for x in pos]
    p = c.pool()
    joint = queries(c, 4, 2, 6 + 2 + 2)
    q = joint[:, :, :6]
    assert not q.is_contiguous()
    keep = p.tensors[0].clone()
    whole = torch.full((6, 2, 6, 128), 3.0, dtype=c.dt, device=DEV)
    for layer in range(3):
        out = run(p, c, seqs, pos, q, [1, 1, 1, 1], layer, whole[1:5])
        want, tol = definition(c, seqs, pos, q, layer)
        assert bool(((out.double() - want).abs() <= tol).all())
    assert bool((whole[0] == 3.0).all()) and bool((whole[5] == 3.0).all()) and bool((p.tensors[0] == keep).all())


def test_a_plan_serves_every_layer_and_another_stream():
    import torch
    c = Cache(4, 64, 1, seed=9, layers=2)
    base = [c._new(PAGE) for _ in range(5)]
    pos = [160 + i for i in range(9)]
    seqs = [c.sequence(x + 1, base) for x in pos]
    p = c.pool()
    q = queries(c, 9, 1, 8)
    n, hq = 9, 8
    size = V.vlac_attend_workspace_bytes(p, n, 1, hq)
    ws = torch.full((size + 64,), 0x5A, dtype=torch.uint8, device=DEV)
    out = torch.zeros((2, n, 1, hq, 64), dtype=c.dt, device=DEV)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        V.vlac_attend_plan(p, i32(seqs), i32(pos), n, 1, hq, None, ws[:size])
        for layer in (1, 0):
            V.vlac_attend_shared(p, layer, n, 1, hq, q, out[layer], ws[:size])
    torch.cuda.current_stream().wait_stream(side)
    for layer in range(2):
        want, tol = definition(c, seqs, pos, q, layer)
        assert bool(((out[layer].double() - want).abs() <= tol).all())
    assert bool((ws[size:] == 0x5A).all())


def test_pages_beyond_32_bit_offsets():
    """A pool of more than 4 GiB: 2^31 values, pages at both ends."""
    import torch
    hq, hkv, hd, layers = 8, 8, 128, 32                       # a page is 4 MiB
    n_pages = 1100
    p = V.new_pages(layers, hkv, hd, 1, n_pages, 4, 4, DEV)
    data, refs, table, length, _ = p.tensors
    c = Cache(hkv, hd, 1, seed=10, layers=layers)
    s = c.sequence(90)
    where = [n_pages - 1, 0, n_pages - 2]
    small = c.pool(extra_seqs=0)
    old = small.tensors[2][0].tolist()
    for j in range(3):
        data[where[j]] = small.tensors[0][old[j]]
    table[1, :3] = i32(where)
    refs[i32(where).long()] = 1
    length[1] = 90
    q = queries(c, 1, 1, hq)
    want, tol = definition(c, [s], [89], q, layers - 1)
    got = run(p, c, [1], [89], q, None, layers - 1)
    assert bool(((got.double() - want).abs() <= tol).all())
    V.vlac_pages_fork(p, i32([1]), i32([2]), 1, True)
    assert table[2].tolist() == [1, 2, 3, -1]
    got2 = run(p, c, [2], [89], q, None, layers - 1)
    assert bool((got2 == got).all())


def test_a_workspace_without_its_plan_is_not_used():
    import torch
    c = Cache(2, 64, 1, seed=11, layers=2)
    base = [c._new(PAGE) for _ in range(2)]
    pos = [70, 75, 66]
    seqs = [c.sequence(x + 2, base) for x in pos]
    p, other = c.pool(), c.pool(seed=1)
    q = queries(c, 3, 2, 4)
    ws = torch.full((V.vlac_attend_workspace_bytes(p, 64, 2, 4),), 0xA5, dtype=torch.uint8, device=DEV)
    out = torch.full((3, 2, 4, 64), 7.0, dtype=c.dt, device=DEV)

    def attend(pool=p, n=3, tokens=2, hq=4):
        rows = n * tokens * hq * 64
        V.vlac_attend_shared(pool, 0, n, tokens, hq, q.view(-1)[:rows].view(n, tokens, hq, 64),
                             out.view(-1)[:rows].view(n, tokens, hq, 64), ws)
        return V.vlac_pages_check(pool, check=False)

    assert attend() == E_RANGE                                  # never planned
    V.vlac_attend_plan(p, i32(seqs), i32(pos), 3, 2, 4, None, ws)
    assert attend(pool=other) == E_RANGE and attend(n=2) == E_RANGE and attend(tokens=1) == E_RANGE and attend(hq=2) == E_RANGE
    assert bool((out == 7.0).all())
    assert attend() == OK
    want, tol = definition(c, seqs, pos, q)
    assert bool(((out.double() - want).abs() <= tol).all())
    V.vlac_attend_plan(other, i32(seqs), i32(pos), 3, 2, 4, None, ws)
    out.fill_(7.0)
    assert attend() == E_RANGE and bool((out == 7.0).all())
    assert attend(pool=other) == OK and bool(((out.double() - want).abs() <= tol).all())
