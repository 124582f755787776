"""Pages at the ends of what is allowed: offsets beyond 32 bits for every call that moves values, as many entries as a
list may hold, and two pools in use at once on two streams."""
import pytest

import paper_2502_02175_amd as V
from pages_model import OK, PAGE, k_tile_at, v_tile_at
from test_gpu_attend import Cache, compare, definition, i32, queries

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def test_append_and_compact_beyond_32_bit_offsets():
    """A pool of 4.3 GiB (2^31 values and more), one sequence in its last two pages."""
    import torch
    layers, heads, hd, n_pages, T = 32, 8, 128, 1100, 37
    p = V.new_pages(layers, heads, hd, 1, n_pages, 2, 3, DEV)
    data, refs, table, length, _ = p.tensors
    far = [n_pages - 1, n_pages - 2]
    data[i32(far + [0, 1]).long()] = 0x5A
    table[1, :2] = i32(far)
    refs[i32(far).long()] = 1
    length[1] = 40
    g = torch.Generator(device=DEV)
    g.manual_seed(1)
    k, v = (torch.randn((1, T, heads, hd), generator=g, device=DEV).half() for _ in range(2))
    V.vlac_pages_append(p, layers - 1, i32([1]), i32([3]), 1, T, k, v)
    live = i32([-7])
    V.vlac_pages_compact(p, live)
    assert V.vlac_pages_check(p, check=False) == OK
    # the last pages, in ascending order, go to the front: n_pages - 2 holds the second 32 positions
    assert live.tolist() == [2] and table[1].tolist() == [1, 0, -1] and refs[:3].tolist() == [1, 1, 0]
    ka, va = (torch.tensor(f(hd), device=DEV) for f in (k_tile_at, v_tile_at))
    d = data.view(torch.int16).view(n_pages, layers, 2, heads, PAGE * hd)
    want = torch.full((2, 2, heads, PAGE * hd), 0x5A5A, dtype=torch.int16, device=DEV)   # [position / 32]
    for t in range(T):
        at = 3 + t
        want[at // PAGE, 0, :, ka[at % PAGE]] = k[0, t].view(torch.int16)
        want[at // PAGE, 1, :, va[at % PAGE]] = v[0, t].view(torch.int16)
    assert bool((d[1, layers - 1] == want[0]).all()) and bool((d[0, layers - 1] == want[1]).all())
    assert bool((d[:2, :layers - 1] == 0x5A5A).all())


def test_attention_of_the_longest_list():
    """4096 entries in groups of one, two, three, ... entries, each with a position of its own."""
    import torch
    n = 4096
    c = Cache(2, 64, 1, seed=2)
    stems = [[c._new(PAGE)] for _ in range(100)]
    group, g = [], 0
    while len(group) < n:
        group += [g] * min(g + 1, n - len(group))
        g += 1
    pos = [32 + (7 * i) % 3 for i in range(n)]
    c_seqs = [c.sequence(pos[i] + 1, stems[group[i]]) for i in range(n)]
    q = queries(c, n, 1, 4)
    compare(c, c.pool(), c_seqs, pos, q, group)


def test_two_pools_at_once_on_two_streams():
    import torch
    runs = []
    for seed in (3, 4):
        c = Cache(4, 64, 1, seed=seed, layers=2)
        base = [c._new(PAGE) for _ in range(6)]
        pos = [192 + i for i in range(7)]
        seqs = [c.sequence(x + 2, base) for x in pos]
        p, q = c.pool(), queries(c, 7, 2, 8)
        ws = torch.empty(V.vlac_attend_workspace_bytes(p, 7, 2, 8), dtype=torch.uint8, device=DEV)
        out = torch.zeros((20, 2, 7, 2, 8, 64), dtype=c.dt, device=DEV)
        runs.append((c, p, q, ws, out, i32(seqs), i32(pos), seqs, pos, torch.cuda.Stream()))
    torch.cuda.synchronize()
    for r in range(20):
        for c, p, q, ws, out, s, at, _, _, stream in runs:
            with torch.cuda.stream(stream):
                V.vlac_attend_plan(p, s, at, 7, 2, 8, None, ws)
                for layer in range(2):
                    V.vlac_attend_shared(p, layer, 7, 2, 8, q, out[r, layer], ws)
    torch.cuda.synchronize()
    for c, p, q, ws, out, _, _, seqs, pos, _ in runs:
        assert bool((out == out[:1]).all())
        for layer in range(2):
            want, tol = definition(c, seqs, pos, q, layer)
            assert bool(((out[0, layer].double() - want).abs() <= tol).all())
