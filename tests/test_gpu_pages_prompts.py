"""Long chunks of new tokens, up to the most that a call may have: rows at the ends and between against the definition in 64 bits,
and every value of an append."""
import random

import pytest

import paper_2502_02175_amd as V
from pages_model import OK, PAGE, k_tile_at, v_tile_at
from test_gpu_attend import Cache, definition, i32, queries, run
from test_gpu_pages import Both, rows

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("n,T,hq,hkv,hd,operand,ahead,group", [
    (1, 4099, 4, 4, 64, 1, [37], None),
    (3, 2500, 12, 2, 128, 0, [0, 64, 1000], None),
    (5, 1031, 8, 8, 128, 1, [2048, 2048, 2100, 0, 31], [0, 0, 0, 1, 1]),
    (1, 65536, 2, 2, 64, 0, [3], None),
    (16, 65536, 2, 1, 64, 1, [0, 33, 4464] + [64 * i for i in range(13)], list(range(16))),   # 2^20 rows
    (16, 65536, 1, 1, 64, 1, [96] * 16, None),
])
def test_rows_of_long_chunks(n, T, hq, hkv, hd, operand, ahead, group):
    import torch
    c = Cache(hkv, hd, operand, seed=n + T)
    s = c.sequence(max(ahead) + T)
    p = c.pool()
    q = torch.empty((n, T, hq, hd), dtype=c.dt, device=DEV)
    for i in range(n):
        q[i] = queries(c, 1, T, hq)[0]
    out = run(p, c, [s] * n, ahead, q, group)
    assert V.vlac_pages_check(p, check=False) == OK
    rng = random.Random(T)
    for i in sorted(set([0, n // 2, n - 1])):
        for t in sorted(set([0, 1, 31, 32, T // 2, T - 2, T - 1] + [rng.randrange(T) for _ in range(9)])):
            want, tol = definition(c, [s], [ahead[i] + t], q[i:i + 1, t:t + 1])
            assert bool(((out[i:i + 1, t:t + 1].double() - want).abs() <= tol).all()), (i, t)
    assert bool(torch.isfinite(out).all())


@pytest.mark.parametrize("n,T,heads,hd,operand", [(1, 5003, 2, 128, 1), (3, 2049, 1, 64, 0), (1, 1 << 17, 1, 64, 1)])
def test_append_of_a_long_chunk(n, T, heads, hd, operand):
    import torch
    dt = torch.bfloat16 if operand == 0 else torch.float16
    columns = (T + 100) // PAGE + 1
    b = Both(n * columns + 3, n + 1, columns, n_kv_heads=heads, head_dim=hd, operand=operand)
    ahead = [5 + 13 * i for i in range(n)]
    for i in range(n):
        b.extend([i], ahead[i])
    pos = i32([0] * n)
    V.vlac_pages_extend(b.p, i32(range(n)), n, T, pos)
    assert pos.tolist() == ahead
    want = b.data.view(torch.int16).view(-1, 2, heads, PAGE * hd).clone()
    k, v = rows(n, T, heads, hd, dt, 1), rows(n, T, heads, hd, dt, 2)
    V.vlac_pages_append(b.p, 0, i32(range(n)), pos, n, T, k, v)
    assert V.vlac_pages_check(b.p, check=False) == OK
    for i in range(n):
        at = ahead[i] + torch.arange(T, device=DEV)
        page = b.table[i, at // PAGE].long()
        for which, x, order in ((0, k, k_tile_at(hd)), (1, v, v_tile_at(hd))):
            place = torch.tensor(order, device=DEV)[at % PAGE]             # [T, hd]
            for h in range(heads):
                want[page[:, None].expand_as(place), which, h, place] = x[i, :, h].view(torch.int16)
    assert bool((b.data.view(torch.int16).view(want.shape) == want).all())
