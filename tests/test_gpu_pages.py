"""Pages of the cache on the GPU: forking, growing, releasing and compacting against the plain model of the pool (every
integer and every value equal), writing of new tokens position by position, importing a stream, graph capture."""
import random

import numpy as np
import pytest

import synth
import paper_2502_02175_amd as V
from pages_model import E_NOMEM, E_RANGE, OK, PAGE, Pool, k_tile_at, pages_of, v_tile_at

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def i32(x):
    import torch
    return torch.tensor(x, dtype=torch.int32, device=DEV)


class Both:
    """A pool on the GPU and its model; a page's values are its first owner's index in every word."""

    def __init__(self, n_pages, max_seqs, max_pages, n_layers=1, n_kv_heads=1, head_dim=64, operand=1):
        import torch
        self.p = V.new_pages(n_layers, n_kv_heads, head_dim, operand, n_pages, max_seqs, max_pages, DEV)
        self.m = Pool(n_pages, max_seqs, max_pages)
        self.data, self.refs, self.table, self.len, self.scratch = self.p.tensors
        self.words = self.data.view(torch.int32).view(n_pages, -1)
        self.words.copy_(torch.arange(n_pages, device=DEV, dtype=torch.int32)[:, None].expand_as(self.words))

    def same(self, where=""):
        assert self.refs.tolist() == self.m.refs, where
        assert self.len.tolist() == self.m.len, where
        assert self.table.tolist() == self.m.table, where
        assert bool((self.words == i32(self.m.data)[:, None]).all()), where
        st = V.vlac_pages_check(self.p, check=False)
        assert st == self.m.check(), where
        assert V.vlac_pages_check(self.p, check=False) == OK           # reported once

    def fork(self, src, dst, deep=False):
        V.vlac_pages_fork(self.p, i32(src), i32(dst), len(src), deep)
        self.m.fork(src, dst, deep)

    def extend(self, seqs, tokens):
        pos = i32([-7] * len(seqs))
        V.vlac_pages_extend(self.p, i32(seqs), len(seqs), tokens, pos)
        assert pos.tolist() == self.m.extend(seqs, tokens)

    def free(self, seqs):
        V.vlac_pages_free(self.p, i32(seqs), len(seqs))
        self.m.free(seqs)

    def compact(self):
        live = i32([-7])
        V.vlac_pages_compact(self.p, live)
        assert live.tolist() == [self.m.compact()]


def test_reset():
    b = Both(70, 9, 5, n_layers=2, n_kv_heads=3)
    b.same()
    b.extend([3, 1], 40)
    b.same()
    V.vlac_pages_reset(b.p)
    b.m = Pool(70, 9, 5)
    b.same()


@pytest.mark.parametrize("seed,n_pages,max_seqs,max_pages,heads,hd,most", [
    (0, 12, 5, 4, 1, 64, 4), (1, 40, 16, 6, 3, 64, 12), (2, 300, 40, 9, 1, 128, 30), (3, 5000, 60, 130, 1, 64, 40),
    (4, 9000, 1500, 7, 1, 64, 1300), (5, 1, 2, 1, 1, 64, 3)])
def test_any_order_of_calls_is_the_model(seed, n_pages, max_seqs, max_pages, heads, hd, most):
    """Random calls, entries that do not fit among them (indices out of range, the same sequence twice, a destination that
    is a source), with and without room."""
    rng = random.Random(seed)
    b = Both(n_pages, max_seqs, max_pages, n_kv_heads=heads, head_dim=hd)
    any_seq = lambda: rng.choice([rng.randrange(max_seqs)] * 12 + [-1, max_seqs, -2 ** 31, 2 ** 31 - 1])
    for step in range(60):
        what = rng.choice(["extend", "extend", "fork", "fork", "deep", "free", "compact"])
        n = rng.choice([1, 2, rng.randint(1, most)])
        seqs = rng.sample(range(max_seqs), min(n, max_seqs)) if rng.random() < 0.5 else [any_seq() for _ in range(n)]
        if what == "extend":
            b.extend(seqs, rng.choice([1, 3, 31, 32, 33, PAGE * rng.randint(1, max_pages)]))
        elif what == "free":
            b.free(seqs)
        elif what == "compact":
            b.compact()
        else:
            src = [any_seq() for _ in seqs] if rng.random() < 0.3 else [rng.randrange(max_seqs) for _ in seqs]
            if rng.random() < 0.7:                              # one or two sources, none of them written
                src = [rng.choice(src[:2]) for _ in src]
                seqs = [s if s not in src else any_seq() for s in seqs]
            b.fork(src, seqs, what == "deep")
        b.same("step %d: %s" % (step, what))


def test_too_few_pages_change_nothing():
    b = Both(9, 6, 8)
    b.extend([0], 100)                                        # 4 pages
    b.extend([1], 33)                                         # 2
    b.same()
    b.fork([0, 0, 0, 0], [2, 3, 4, 1])                       # 4 last pages wanted, 3 and the 2 released: there is room
    b.same()
    b.fork([0], [5], deep=True)
    assert b.m.full
    b.same()
    b.extend([0, 2], 33)                                      # (one would have fitted)
    b.extend([0], 28)
    b.same()


def test_forking_over_a_continuation_of_the_same_source_is_repeatable():
    b = Both(30, 6, 8)
    b.extend([5], 75)
    for _ in range(3):
        b.fork([5, 5, 5], [0, 1, 2])
        b.same()
        assert b.m.table[0][:3] == [0, 1, 3] and b.m.refs[:3] == [4, 4, 1]


def test_lists_of_the_largest_size():
    n = 4096
    b = Both(3 * n, 2 * n, 2)
    b.extend(list(range(n)), 17)
    b.same()
    b.fork(list(range(n)), list(range(n, 2 * n)))
    b.same()
    b.free(list(range(0, 2 * n, 2)))
    b.compact()
    b.same()


# ---- values of new tokens ----

def rows(n, T, heads, hd, dt, seed):
    import torch
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return torch.randint(-2 ** 15, 2 ** 15, (n, T, heads, hd), generator=g, device=DEV, dtype=torch.int16).view(dt)  # NaN among them


@pytest.mark.parametrize("heads,hd,operand,T", [(4, 64, 1, 1), (2, 128, 0, 1), (3, 64, 0, 5), (1, 128, 1, 67), (32, 128, 1, 2),
                                               (5, 64, 2, 33)])
def test_append_writes_exactly_its_positions(heads, hd, operand, T):
    import torch
    dt = torch.bfloat16 if operand == 0 else torch.float16
    L, n = 3, 40                                               # entries at every offset of a page
    b = Both(300, n + 4, 6, n_layers=L, n_kv_heads=heads, head_dim=hd, operand=operand)
    order = random.Random(1).sample(range(n + 4), n)
    for k in range(n):
        b.extend([order[k]], 1 + k % 33)
    pos = i32([0] * n)
    V.vlac_pages_extend(b.p, i32(order), n, T, pos)
    want = b.data.view(torch.int16).view(300, L, 2, heads, PAGE * hd).clone()
    table, at = b.table.cpu().numpy(), pos.cpu().numpy()
    ka, va = torch.tensor(k_tile_at(hd), device=DEV), torch.tensor(v_tile_at(hd), device=DEV)
    pos[7] = -1                                                # skipped, and no error
    joint = rows(n, T, 2 * heads + 3, hd, dt, 5)               # (slices of a joint projection)
    for layer in (1, 2):
        k, v = (joint[:, :, :heads], joint[:, :, heads:2 * heads]) if layer == 1 else \
            (rows(n, T, heads, hd, dt, 6), rows(n, T, heads, hd, dt, 7))
        V.vlac_pages_append(b.p, layer, i32(order), pos, n, T, k, v)
        for i in range(n):
            if i == 7:
                continue
            for t in range(T):
                page, r = table[order[i]][(at[i] + t) // PAGE], (at[i] + t) % PAGE
                want[page, layer, 0, :, ka[r]] = k[i, t].view(torch.int16)
                want[page, layer, 1, :, va[r]] = v[i, t].view(torch.int16)
    got = b.data.view(torch.int16).view(want.shape)
    assert bool((got == want).all())
    assert V.vlac_pages_check(b.p, check=False) == OK


def test_append_keeps_out_of_shared_pages_and_out_of_range():
    import torch
    b = Both(40, 8, 4, n_kv_heads=2)
    b.extend([0], 70)
    b.fork([0], [1])
    b.extend([1], 3)                                           # positions 70..72 on its own page
    before = b.data.clone()
    k = rows(1, 2, 2, 64, torch.float16, 1)

    def refused(seq, pos):
        V.vlac_pages_append(b.p, 0, i32([seq]), i32([pos]), 1, 2, k, k)
        assert V.vlac_pages_check(b.p, check=False) == E_RANGE, (seq, pos)
        assert bool((b.data == before).all()), (seq, pos)

    refused(1, 10)                                            # a page that sequence 0 holds too
    refused(0, 62)
    refused(1, 73)                                            # behind the end
    refused(5, 0)                                             # empty
    refused(8, 0)
    refused(-1, 0)
    refused(1, 2 ** 31 - 1)
    V.vlac_pages_append(b.p, 0, i32([1]), i32([72]), 1, 2, k, k)   # one position inside, one behind the end
    assert V.vlac_pages_check(b.p, check=False) == E_RANGE
    table = b.table.cpu().numpy()
    changed = (b.data != before).any(1).nonzero().flatten().tolist()
    assert changed == [table[1][2]]


def test_binding_checks_of_rows_and_lists():
    import torch
    b = Both(40, 8, 4, n_kv_heads=2)
    good = torch.zeros((2, 3, 2, 64), dtype=torch.float16, device=DEV)
    call = lambda k, v, seqs=i32([0, 1]), pos=i32([0, 0]): V.vlac_pages_append(b.p, 0, seqs, pos, 2, 3, k, v)
    with pytest.raises(TypeError):
        call(good.bfloat16(), good.bfloat16())
    with pytest.raises(ValueError):
        call(good[:1], good[:1])                               # too few rows
    with pytest.raises(ValueError):
        call(good.transpose(1, 2).contiguous().transpose(1, 2), good)   # heads outermost: rows are not dense
    with pytest.raises(ValueError):
        call(good, torch.zeros((2, 3, 4, 64), dtype=torch.float16, device=DEV)[:, :, :2])   # two strides
    with pytest.raises(ValueError):
        call(good, good, seqs=i32([0]))
    with pytest.raises(TypeError):
        call(good, good, pos=i32([0, 0]).long())
    with pytest.raises(ValueError):
        call(good.cpu(), good.cpu())
    with pytest.raises(V.VlacError):
        call(torch.zeros((1, 1, 2, 64), dtype=torch.float16, device=DEV).expand(2, 3, 2, 64),
             torch.zeros((1, 1, 2, 64), dtype=torch.float16, device=DEV).expand(2, 3, 2, 64))   # rows on top of each other


# ---- a prefill's cache ----

@pytest.mark.parametrize("operand,L", [("f16", 64), ("bf16", 47), ("f16w8", 33)])
def test_import_takes_the_tiles_of_the_streams(operand, L):
    import torch
    from helpers import GpuModel
    cfg = synth.CONFIGS["tiny"]
    gm = GpuModel(cfg, seed=2, max_batch=3, max_seq=96, operand=operand)
    try:
        rng = np.random.default_rng(3)
        mine = V.new_pages(cfg.n_layers, cfg.n_kv_heads, cfg.head_dim, gm.ccfg.operand_dtype, 20, 6, 3, DEV)
        data, refs, table, length, _ = mine.tensors
        data.fill_(0x5A)
        seqs = i32([4, 0, 5])
        assert V.vlac_pages_import(gm.ctx, gm.kv, 3, L, mine, seqs, check=False) == -4       # nothing there yet
        gm.prefill(synth.round_bf16(rng.standard_normal((3, L, cfg.d_model))), L - 16, want_stats=False)
        pos = i32([0])
        V.vlac_pages_extend(mine, i32([0]), 1, 40, pos)                                       # (released again)
        V.vlac_pages_import(gm.ctx, gm.kv, 3, L, mine, seqs)
        n = pages_of(L)
        want = [[-1] * 3 for _ in range(6)]
        for k, s in enumerate((4, 0, 5)):
            want[s][:n] = range(k * n, k * n + n)
        assert table.tolist() == want and refs.tolist() == [1] * (3 * n) + [0] * (20 - 3 * n)
        assert length.tolist() == [L, 0, 0, 0, L, L]
        cache = gm.kv.view(torch.int16).view(3, cfg.n_layers, 2, cfg.n_kv_heads, 3, PAGE * cfg.head_dim)
        got = data.view(torch.int16).view(20, cfg.n_layers, 2, cfg.n_kv_heads, PAGE * cfg.head_dim)
        for k in range(3):
            for j in range(n):
                assert bool((got[k * n + j] == cache[k, :, :, :, j]).all()), (k, j)
        assert bool((data[3 * n:] == 0x5A).all())
        V.vlac_pages_import(gm.ctx, gm.kv, 2, L, mine, i32([1, 1]))                          # the second is ignored
        assert V.vlac_pages_check(mine, check=False) == E_RANGE and length.tolist() == [L, L, 0, 0, L, L]
        bad = lambda L=L, B=3, p=mine, s=seqs: V.vlac_pages_import(gm.ctx, gm.kv, B, L, p, s, check=False)
        assert bad(L=97) == -2 and bad(L=0) == -3 and bad(B=0) == -3 and bad(B=4, s=i32([0, 1, 2, 3])) == -3 and bad(s=None) == -1
        other = V.new_pages(cfg.n_layers, cfg.n_kv_heads, cfg.head_dim, 1 - (gm.ccfg.operand_dtype > 0), 20, 6, 3, DEV)
        assert bad(p=other) == -2
        small = V.new_pages(cfg.n_layers, cfg.n_kv_heads, cfg.head_dim, gm.ccfg.operand_dtype, n, 6, 3, DEV)
        V.vlac_pages_import(gm.ctx, gm.kv, 3, L, small, seqs)
        assert V.vlac_pages_check(small, check=False) == E_NOMEM and small.tensors[3].tolist() == [0] * 6
    finally:
        gm.close()


# ---- capture ----

def test_a_captured_turn_replays_like_the_eager_one():
    """Fork, room, new tokens, attention and release in one graph, replayed between eager work on another pool."""
    import torch
    torch.manual_seed(0)
    heads, hd, T, n = 2, 64, 3, 5
    b = Both(60, 12, 8, n_kv_heads=heads, head_dim=hd)
    b.data.view(torch.float16).copy_(torch.randn(b.data.view(torch.float16).shape, device=DEV).half())
    b.extend([0], 75)
    src, dst = i32([0] * n), i32([1, 2, 3, 4, 7])
    pos, live = i32([0] * n), i32([0])
    k, v = (torch.randn((n, T, heads, hd), device=DEV).half() for _ in range(2))
    q, out = torch.randn((n, T, 6, hd), device=DEV).half(), torch.zeros((n, T, 6, hd), device=DEV, dtype=torch.float16)
    ws = torch.empty(V.vlac_attend_workspace_bytes(b.p, n, T, 6), dtype=torch.uint8, device=DEV)

    def turn():
        V.vlac_pages_fork(b.p, src, dst, n)
        V.vlac_pages_extend(b.p, dst, n, T, pos)
        V.vlac_pages_append(b.p, 0, dst, pos, n, T, k, v)
        V.vlac_attend_plan(b.p, dst, pos, n, T, 6, src, ws)
        V.vlac_attend_shared(b.p, 0, n, T, 6, q, out, ws)
        V.vlac_pages_free(b.p, dst, n)
        V.vlac_pages_compact(b.p, live)

    turn()
    torch.cuda.synchronize()
    eager = out.clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        turn()
    torch.cuda.current_stream().wait_stream(side)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        turn()
    for r in range(4):
        k.copy_(torch.randn_like(k))
        q.copy_(torch.randn_like(q))
        turn()
        torch.cuda.synchronize()
        eager.copy_(out)
        state = [x.clone() for x in b.p.tensors]
        out.zero_()
        g.replay()
        other = Both(20, 4, 4)                                  # eager work of its own between the replays
        other.extend([0, 1], 40)
        other.same()
        torch.cuda.synchronize()
        assert bool((out == eager).all()), r
        for x, y in zip(b.p.tensors[:4], state):
            assert bool((x == y).all()), r
        assert V.vlac_pages_check(b.p, check=False) == OK
