"""Keys and values appended with norm and rotation on the way, against the definition in 64 bits: head layouts, both pairings, parts
of a head, scaled tables, far places, trees' places, strided and in-place rows; what is not written stays as it was, bit for bit."""
import math

import pytest

import paper_2502_02175_amd as V
from pages_model import E_RANGE, OK, PAGE, k_tile_at, pages_of, v_tile_at

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def i32(x):
    import torch
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def table_of(dims, base, factor, original, low, high):
    """Turns per position, in Python's doubles."""
    out = []
    for f in range(dims // 2):
        w = base ** (-2.0 * f / dims) / (2 * math.pi)
        r = original * w
        keep = 0.0 if original == 0 or r <= low else 1.0 if r >= high else (r - low) / (high - low)
        out.append(w * (keep + (1 - keep) / factor))
    return out


@pytest.mark.parametrize("dims", [2, 6, 64, 128])
@pytest.mark.parametrize("base,factor,original,low,high", [(1e4, 1, 0, 1, 32), (5e5, 4, 0, 1, 4), (1e4, 8, 8192, 1, 4), (1e6, 2.5, 100, 0, 32)])
def test_the_table(dims, base, factor, original, low, high):
    import torch
    r = V.rotary(dims, V.ROTARY_HALF, base, factor, original, low, high)
    want = torch.tensor(table_of(dims, base, factor, original, low, high), dtype=torch.float64)
    # a power (2 steps), five products, quotients and sums
    assert bool(((r.tensors[0].cpu() / want - 1).abs() <= 16 * 2.0 ** -53).all())


class Setup:
    """Sequences of a pool of random bits (finite values), each with room for `tokens` new positions at its end."""

    def __init__(self, hkv, hd, operand, starts, tokens, layers=2, seed=0, max_pages=None):
        import torch
        self.hkv, self.hd, self.layers, self.tokens = hkv, hd, layers, tokens
        self.dt = torch.bfloat16 if operand == 0 else torch.float16
        self.g = torch.Generator(device=DEV)
        self.g.manual_seed(seed)
        held = [pages_of(x + tokens) for x in starts]
        self.n_pages = sum(held) + 3
        self.pool = V.new_pages(layers, hkv, hd, operand, self.n_pages, len(starts) + 2, max_pages or max(held) + 1, DEV)
        data, refs, table, length, _ = self.pool.tensors
        self.data = data.view(torch.int16).view(self.n_pages, layers, 2, hkv, PAGE * hd)
        self.data.copy_(self.randn(self.data.shape).view(torch.int16))
        order = torch.randperm(self.n_pages, generator=self.g, device=DEV).tolist()
        self.table = []
        for s, k in enumerate(held):
            mine, order = order[:k], order[k:]
            table[s, :k] = i32(mine)
            refs[torch.tensor(mine, device=DEV)] = 1
            self.table.append(mine)
        length[:len(starts)] = i32([x + tokens for x in starts])
        self.seqs, self.pos = list(range(len(starts))), list(starts)

    def randn(self, shape, scale=1.0):
        import torch
        return (scale * torch.randn(shape, generator=self.g, device=DEV)).to(self.dt)

    def rows(self, data, which, layer, s, at):
        """K (0) or V (1) of sequence s at positions `at`, [len(at), hkv, hd]."""
        import torch
        tile = torch.tensor((k_tile_at, v_tile_at)[which](self.hd), device=DEV)
        x = [data[self.table[s][p // PAGE], layer, which][:, tile[p % PAGE]] for p in at]
        return torch.stack(x).view(self.dt)

    def masked(self, layer, written):
        """The pool's bits with what may have been written taken out."""
        import torch
        keep = torch.ones(self.data.shape, dtype=torch.bool, device=DEV)
        for s, p in written:
            for which, f in ((0, k_tile_at), (1, v_tile_at)):
                keep[self.table[s][p // PAGE], layer, which][:, torch.tensor(f(self.hd)[p % PAGE], device=DEV)] = False
        return keep


def definition(x, places, rot, gain, eps):
    """x [n, T, heads, hd] -> R(place) N(x) in 64 bits, and how far fp32 may be from it before the last rounding."""
    import torch
    hd = x.shape[-1]
    y = x.double()
    rel = 0.0
    if gain is not None:
        y = y / torch.sqrt((y * y).mean(-1, keepdim=True) + eps) * gain.double()
        # hd products and sums of one sign, the mean, eps (each half a step; the root halves them), the root, two products
        rel = ((hd + 4) / 2 + 2 + 2) * 2.0 ** -24
    err = rel * y.abs()
    if rot is None:
        return y, err
    dims, pairs, amp, turns = rot
    f = torch.arange(dims, device=DEV)
    half = dims // 2
    pair, second = (f // 2, f % 2 == 1) if pairs else (f % half, f >= half)
    other = torch.where(second, f - 1, f + 1) if pairs else torch.where(second, f - half, f + half)
    t = places.double()[:, :, None] * turns.double()[pair]
    angle = 2 * math.pi * (t - torch.floor(t))[:, :, None, :]
    co, si = torch.cos(angle) * amp, torch.sin(angle) * amp
    a, b = y[..., :dims], y[..., other]
    z = y.clone()
    z[..., :dims] = torch.where(second, a * co + b * si, a * co - b * si)
    # the turn in 64 bits, its fraction in 32, the chip's sine and cosine (1.26e-7 over a turn), the amplitude, two products and a sum
    trig = 2 * math.pi * (2.0 ** -25 + t.abs().amax().item() * 2.0 ** -52) + 1.26e-7 + 2.0 ** -23
    e = err.clone()
    e[..., :dims] = (a.abs() + b.abs()) * abs(amp) * (rel + trig + 2 * 2.0 ** -24)
    return z, e


def near(got, want, err, dt):
    import torch
    half = torch.finfo(dt).eps / 2
    tol = err * (1 + half) + half * want.abs() + torch.finfo(dt).tiny * half * 2
    off = (got.double() - want).abs()
    assert bool(torch.isfinite(got).all())
    assert bool((off <= tol).all()), "%.3g over the bound" % float((off / tol).max())


LAYOUTS = [(4, 4, 64), (12, 2, 128), (1, 1, 128), (16, 4, 64), (3, 5, 128)]


def call(s, layer, rot, places, hq, q, k, v, out, gains, eps=1e-5, pos=None, seqs=None):
    n = len(s.seqs if seqs is None else seqs)
    V.vlac_pages_append_rotated(s.pool, layer, i32(s.seqs if seqs is None else seqs), i32(s.pos if pos is None else pos), n, s.tokens, rot,
                                places, hq, q, k, v, out, *gains, eps)


@pytest.mark.parametrize("hq,hkv,hd", LAYOUTS)
@pytest.mark.parametrize("operand", [0, 1])
@pytest.mark.parametrize("layout,dims,norm,tokens", [
    (V.ROTARY_HALF, "all", "qk", 1), (V.ROTARY_HALF, "all", "", 31), (V.ROTARY_PAIRS, "all", "k", 9), (V.ROTARY_HALF, 2, "q", 8),
    (V.ROTARY_HALF, 22, "qk", 17), (V.ROTARY_PAIRS, 6, "", 40), (V.ROTARY_HALF, 48, "", 3), (V.ROTARY_PAIRS, 62, "qk", 70),
    (None, 0, "qk", 5)])
def test_against_the_definition(hq, hkv, hd, operand, layout, dims, norm, tokens):
    import torch
    starts = [0, 7, 31, 32, 90, 301]
    s = Setup(hkv, hd, operand, starts, tokens, seed=hd + tokens)
    n, d = len(starts), hd if dims == "all" else dims
    rot = None if layout is None else V.rotary(d, layout, 1e4, 4.0, 64, 1.0, 4.0, amplitude=1.25)
    qkv = s.randn((n, tokens, hq + 2 * hkv, hd), 2.0)          # rows of a joint projection
    q, k, v = qkv.split((hq, hkv, hkv), 2)
    gains = [(1 + 0.3 * torch.randn(hd, generator=s.g, device=DEV)).bfloat16() if w in norm else None for w in "qk"]
    out = torch.full((n, tokens, hq, hd), 7.0, dtype=s.dt, device=DEV)
    before, given = s.data.clone(), qkv.clone()
    call(s, 1, rot, None, hq, q, k, v, out, gains)
    assert V.vlac_pages_check(s.pool, check=False) == OK and torch.equal(qkv.view(torch.int16), given.view(torch.int16))
    places = torch.tensor([[p + t for t in range(tokens)] for p in starts], device=DEV)
    spec = None if rot is None else (d, layout == V.ROTARY_PAIRS, 1.25, rot.tensors[0])
    for x, gain, got in ((q, gains[0], out), (k, gains[1], None)):
        want, err = definition(x, places, spec, gain, 1e-5)
        if got is None:
            got = torch.stack([s.rows(s.data, 0, 1, i, range(p, p + tokens)) for i, p in enumerate(starts)])
        near(got, want, err, s.dt)
        if gain is None:                                       # features beyond the rotated ones are copies
            assert torch.equal(got[..., d:].contiguous().view(torch.int16), x[..., d:].contiguous().view(torch.int16))
    for i, p in enumerate(starts):
        assert torch.equal(s.rows(s.data, 1, 1, i, range(p, p + tokens)), v[i])
    keep = s.masked(1, [(i, p + t) for i, p in enumerate(starts) for t in range(tokens)])
    assert torch.equal(s.data[keep], before[keep])
    # the same bits again; queries in place; without queries
    after = s.data.clone()
    call(s, 1, rot, None, hq, q, k, v, q, gains)
    assert torch.equal(q.contiguous().view(torch.int16), out.view(torch.int16)) and torch.equal(s.data, after)
    s.data.copy_(before)
    call(s, 1, rot, None, 0, None, k, v, None, gains)
    assert torch.equal(s.data, after)


@pytest.mark.parametrize("hq,hkv,hd,n,tokens", [(31, 6, 64, 5, 200), (30, 7, 128, 3, 601), (9, 2, 128, 80, 33), (5, 2, 64, 3, 3400),
                                                   (1, 13, 128, 300, 9)])
@pytest.mark.parametrize("operand", [0, 1])
@pytest.mark.parametrize("layout,dims,norm", [(V.ROTARY_HALF, 64, "qk"), (V.ROTARY_PAIRS, 64, ""), (V.ROTARY_HALF, 50, "k"), (None, 0, "q")])
def test_calls_whose_waves_take_several_heads(hq, hkv, hd, n, tokens, operand, layout, dims, norm):
    """4096 and 8192 heads of 8 positions and more; numbers of heads that the waves do not divide."""
    import torch
    assert n * ((tokens + 14) // 8) * (hq + hkv) >= 4096
    starts = [(37 * i + 5) % 90 for i in range(n)]
    s = Setup(hkv, hd, operand, starts, tokens, layers=1, seed=tokens)
    rot = None if layout is None else V.rotary(dims, layout, 1e4)
    qkv = s.randn((n, tokens, hq + 2 * hkv, hd))
    q, k, v = qkv.split((hq, hkv, hkv), 2)
    gains = [(1 + 0.3 * torch.randn(hd, generator=s.g, device=DEV)).bfloat16() if w in norm else None for w in "qk"]
    out = torch.empty((n, tokens, hq, hd), dtype=s.dt, device=DEV)
    before = s.data.clone()
    call(s, 0, rot, None, hq, q, k, v, out, gains)
    assert V.vlac_pages_check(s.pool, check=False) == OK
    places = torch.tensor(starts, device=DEV)[:, None] + torch.arange(tokens, device=DEV)
    table = s.pool.tensors[2].long()
    page, r = table[torch.arange(n, device=DEV)[:, None], places // PAGE], places % PAGE
    ka, va = (torch.tensor(f(hd), device=DEV)[r] for f in (k_tile_at, v_tile_at))          # [n, tokens, hd]
    kk, vv = (torch.gather(s.data[:, 0, w][page], 3, at[:, :, None, :].expand(-1, -1, hkv, -1)).view(s.dt) for w, at in ((0, ka), (1, va)))
    assert torch.equal(vv, v)
    spec = None if rot is None else (dims, layout == V.ROTARY_PAIRS, 1.0, rot.tensors[0])
    for x, gain, got in ((q, gains[0], out), (k, gains[1], kk)):
        want, err = definition(x, places, spec, gain, 1e-5)
        near(got, want, err, s.dt)
    again = s.data.clone()                                      # nothing else was written
    for w, at in ((0, ka), (1, va)):
        again[:, 0, w][page[..., None, None], torch.arange(hkv, device=DEV)[:, None], at[:, :, None, :]] = \
            before[:, 0, w][page[..., None, None], torch.arange(hkv, device=DEV)[:, None], at[:, :, None, :]]
    assert torch.equal(again, before)
    call(s, 0, rot, None, hq, q, k, v, q, gains)                # in place
    assert torch.equal(q.contiguous().view(torch.int16), out.view(torch.int16))


@pytest.mark.parametrize("operand,hd", [(1, 128), (0, 64)])
@pytest.mark.parametrize("layout", [V.ROTARY_HALF, V.ROTARY_PAIRS])
def test_places_of_its_own(operand, hd, layout):
    """Far places (their angles need 64 bits), repeated ones, and rows that are not there: zeros."""
    import torch
    s = Setup(2, hd, operand, [5, 64], 6, seed=3)
    places = [[0, 1, 1, -1, 1000003, 2 ** 31 - 1], [-2, 77, -1, 32767, 131071, 16777217]]
    rot = V.rotary(hd, layout, 5e5)
    q, k, v = s.randn((2, 6, 4, hd)), s.randn((2, 6, 2, hd)), s.randn((2, 6, 2, hd))
    k[0, 3] = v[0, 3] = q[0, 3] = float("nan")                 # (nothing to be read there)
    out = torch.full_like(q, 7.0)
    call(s, 0, rot, i32(places), 4, q, k, v, out, (None, None))
    at = torch.tensor(places, device=DEV)
    gone = at < 0
    spec = (hd, layout == V.ROTARY_PAIRS, 1.0, rot.tensors[0])
    kk = torch.stack([s.rows(s.data, 0, 0, i, range(p, p + 6)) for i, p in enumerate(s.pos)])
    vv = torch.stack([s.rows(s.data, 1, 0, i, range(p, p + 6)) for i, p in enumerate(s.pos)])
    for got, x in ((out, q), (kk, k)):
        want, err = definition(torch.where(gone[:, :, None, None], torch.zeros_like(x), x), at, spec, None, 0)
        near(got, want, err, s.dt)
    for got in (out, kk, vv):
        assert not bool(got[gone].any())
    assert torch.equal(vv[~gone], v[~gone])


def test_values_at_the_ends_of_the_type():
    """fp16: a finite result beyond the range saturates, infinities and NaN stay what they are and where they are; unrotated features
    and heads without norm are copies."""
    import torch
    s = Setup(1, 64, 1, [3], 4, seed=5)
    rot = V.rotary(32, V.ROTARY_HALF, 1e4)
    x = s.randn((1, 4, 1, 64))
    x[0, 0, 0, 0], x[0, 0, 0, 16] = 65504.0, -65504.0          # turned beyond the range
    x[0, 1, 0, 40], x[0, 1, 0, 41], x[0, 1, 0, 42] = float("inf"), float("-inf"), float("nan")
    x[0, 2, 0, 5] = float("inf")
    x[0, 3, 0, 50] = 2.0 ** -24
    out = torch.zeros_like(x)
    call(s, 0, rot, i32([[1, 4, 5, 6]]), 1, x, x, x, out, (None, None))
    k, v = (s.rows(s.data, w, 0, 0, range(3, 7)) for w in (0, 1))
    assert torch.equal(v.view(torch.int16), x[0].view(torch.int16))
    assert torch.equal(out[0].view(torch.int16), k.view(torch.int16))
    y = out[0, :, 0]
    assert torch.equal(y[:, 32:].contiguous().view(torch.int16), x[0, :, 0, 32:].contiguous().view(torch.int16))
    c, w = math.cos(1.0), math.sin(1.0)
    assert 65504 * (c + w) > 65504 and float(y[0, 0]) == 65504.0
    assert abs(float(y[0, 16]) - 65504 * (w - c)) <= 65504 * 2.0 ** -11
    assert math.isinf(float(y[2, 5])) and not math.isfinite(float(y[2, 21]))
    assert bool(torch.isfinite(y[2, :5]).all()) and bool(torch.isfinite(y[2, 6:21]).all())


def test_entries_that_do_not_fit():
    """Negative positions are skipped; unknown sequences, shared pages and positions behind the sequence are reported, their queries
    are there all the same."""
    import torch
    T = 5
    s = Setup(2, 64, 1, [30, 40, 50, 60], T, seed=6)
    data, refs, table, length, _ = s.pool.tensors
    refs[s.table[2][1]] = 2                                    # positions 50 .. 54 lie in a shared page
    q, k, v = s.randn((5, T, 3, 64)), s.randn((5, T, 2, 64)), s.randn((5, T, 2, 64))
    rot = V.rotary(64, V.ROTARY_HALF, 1e4)
    out = torch.full_like(q, 7.0)
    before = s.data.clone()
    seqs, pos = [0, 1, 2, 99, 3], [30, -1, 50, 10, 62]         # the last one: positions 65, 66 are behind its end
    call(s, 0, rot, None, 3, q, k, v, out, (None, None), pos=pos, seqs=seqs)
    assert V.vlac_pages_check(s.pool, check=False) == E_RANGE and V.vlac_pages_check(s.pool, check=False) == OK
    assert bool((out[1] == 7).all())
    for i in (0, 2, 3, 4):
        want, err = definition(q[i:i + 1], torch.tensor([[pos[i] + t for t in range(T)]], device=DEV), (64, False, 1.0, rot.tensors[0]), None, 0)
        near(out[i:i + 1], want, err, s.dt)
    written = [(0, 30 + t) for t in range(T)] + [(3, 62 + t) for t in range(3)]
    keep = s.masked(0, written)
    assert torch.equal(s.data[keep], before[keep])
    assert torch.equal(s.rows(s.data, 1, 0, 3, (62, 63, 64)), v[4, :3]) and torch.equal(s.rows(s.data, 1, 0, 0, range(30, 35)), v[0])
    assert not torch.equal(s.rows(s.data, 0, 0, 3, (62, 63, 64)), s.rows(before, 0, 0, 3, (62, 63, 64)))
    # a length out of range, a table that names no page
    length[0], table[1, 1] = -3, s.n_pages
    before = s.data.clone()
    call(s, 0, rot, None, 0, None, k[:2], v[:2], None, (None, None), pos=[30, 40], seqs=[0, 1])
    assert V.vlac_pages_check(s.pool, check=False) == E_RANGE and torch.equal(s.data, before)


def test_offsets_beyond_32_bits():
    """The last page of a pool of more than 2^32 values, and rows that lie 2^30 values apart."""
    import torch
    layers, hkv, hd = 32, 32, 128
    n_pages = (1 << 32) // (layers * 2 * hkv * PAGE * hd) + 3
    p = V.new_pages(layers, hkv, hd, 1, n_pages, 1, 1, DEV)
    data, refs, table, length, _ = p.tensors
    table[0, 0], length[0], refs[n_pages - 1] = n_pages - 1, 20, 1
    page = data[n_pages - 1].view(torch.int16).view(layers, 2, hkv, PAGE * hd)
    page.zero_()
    k = torch.randn((1, 3, hkv, hd), device=DEV).half()
    wide = torch.empty((1 << 31) + 4096, dtype=torch.float16, device=DEV)
    q = wide.as_strided((1, 3, 1, hd), (3 << 30, 1 << 30, hd, 1))
    q.copy_(torch.randn((1, 3, 1, hd), device=DEV))
    out = torch.zeros((1, 3, 1, hd), dtype=torch.float16, device=DEV)
    V.vlac_pages_append_rotated(p, layers - 1, i32([0]), i32([17]), 1, 3, None, None, 1, q, k, k, out)
    assert V.vlac_pages_check(p, check=False) == OK
    assert torch.equal(out, q)
    for which, f in ((0, k_tile_at), (1, v_tile_at)):
        at = torch.tensor(f(hd)[17:20], device=DEV)
        assert torch.equal(page[layers - 1, which][:, at].permute(1, 0, 2).contiguous().view(torch.float16), k[0])
        page[layers - 1, which][:, at] = 0
    assert not bool(page.any())


def test_the_longest_list():
    """4096 sequences of one token each."""
    import torch
    n, hkv, hd = 4096, 2, 64
    p = V.new_pages(1, hkv, hd, 0, n, n, 1, DEV)
    data, refs, table, length, _ = p.tensors
    order = torch.randperm(n, device=DEV).int()
    table[:, 0], length[:] = order, 1 + torch.arange(n, device=DEV, dtype=torch.int32) % 32
    refs.fill_(1)
    seqs = torch.randperm(n, device=DEV).int()
    pos = length[seqs.long()] - 1
    q, k, v = (torch.randn((n, 1, h, hd), device=DEV).bfloat16() for h in (3, hkv, hkv))
    rot, out = V.rotary(hd), torch.empty_like(q)
    V.vlac_pages_append_rotated(p, 0, seqs, pos, n, 1, rot, None, 3, q, k, v, out)
    assert V.vlac_pages_check(p, check=False) == OK
    d = data.view(torch.int16).view(n, 2, hkv, PAGE * hd)[order[seqs.long()].long()]
    ka, va = (torch.tensor(f(hd), device=DEV)[pos.long()] for f in (k_tile_at, v_tile_at))
    kk, vv = (torch.gather(d[:, w], 2, at[:, None, :].expand(-1, hkv, -1)).view(torch.bfloat16)[:, None] for w, at in ((0, ka), (1, va)))
    assert torch.equal(vv, v)
    for x, got in ((q, out), (k, kk)):
        want, err = definition(x, pos.long()[:, None], (hd, False, 1.0, rot.tensors[0]), None, 0)
        near(got, want, err, torch.bfloat16)


@pytest.mark.parametrize("hd,layout", [(128, V.ROTARY_HALF), (64, V.ROTARY_PAIRS), (64, None)])
def test_norms_whose_squares_leave_fp32(hd, layout):
    """bf16 has fp32's range: rows of 2^-120 to 2^126, ordinary ones beside them, and an eps that is far below or far above the squares."""
    import torch
    scales = [2.0 ** 126, 2.0 ** 90, 2.0 ** 62, 1.0, 2.0 ** -40, 2.0 ** -62, 2.0 ** -75, 2.0 ** -120]
    s = Setup(2, hd, 0, [9], len(scales), seed=6)
    rot = None if layout is None else V.rotary(hd, layout, 1e4)
    spec = None if rot is None else (hd, layout == V.ROTARY_PAIRS, 1.0, rot.tensors[0])
    up = torch.tensor(scales, device=DEV, dtype=torch.float64)[None, :, None, None]
    draw = lambda heads: ((torch.rand((1, len(scales), heads, hd), generator=s.g, device=DEV, dtype=torch.float64) * 2 - 1) * up).to(s.dt)
    q, k = draw(3), draw(2)
    gains = s.randn((hd,)), s.randn((hd,))
    places = i32([list(range(100, 100 + len(scales)))])
    for eps in (0.0, 2.0 ** -130, 1e-5):
        out = torch.zeros_like(q)
        call(s, 0, rot, places, 3, q, k, k, out, gains, eps=eps)
        kk = s.rows(s.data, 0, 0, 0, range(9, 9 + len(scales)))[None]
        eps32 = torch.tensor(eps, dtype=torch.float32).double().item()
        for got, x, gain in ((out, q, gains[0]), (kk, k, gains[1])):
            want, err = definition(x, places, spec, gain, eps32)
            near(got, want, err, s.dt)
    z = torch.zeros_like(q)
    call(s, 0, rot, places, 3, z, k, k, out, gains, eps=1e-5)
    assert not bool(out.any())
