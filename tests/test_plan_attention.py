"""Host logic without a GPU: how the attention over pages cuts its work (the rules that its plan evaluates on the device, through their
inspection entry point), and that what comes of it has room in the workspace that the host sizes without the lists."""
import ctypes as C
import random

import pytest

import paper_2502_02175_amd as V
from pages_model import PAGE

POOL = dict(n_layers=1, head_dim=64, operand_dtype=0, n_pages=1 << 20, max_seqs=4096)


def pool(hkv, max_pages):
    return V.Pages(POOL["n_layers"], hkv, POOL["head_dim"], POOL["operand_dtype"], POOL["n_pages"], POOL["max_seqs"], max_pages)


def plan(hq, hkv, n, pages, tokens=1, group=None, max_pages=None, behind=0):
    """n entries, `pages` pages in common, the new tokens `behind` positions further."""
    pos = [pages * PAGE + behind] * n
    if max_pages is None:
        max_pages = min(-(-(pos[0] + tokens) // PAGE), 32768)
    return V.vlac_plan_attention(pool(hkv, max_pages), tokens, hq, pos, group, [pages] * n)


def fits(x):
    cols, (items, items_room), (parts, parts_room) = x
    assert 0 < items <= items_room and 0 <= parts <= parts_room, x
    return cols


LENGTHS = [65, 66, 100, 127, 128, 129, 257, 1000, 1025, 3257, 5692, 6000, 9123, 16384, 32000, 32767]


@pytest.mark.parametrize("heads", [(1, 1), (2, 1), (4, 1), (8, 1), (16, 1), (17, 1), (2, 2), (4, 2), (12, 2), (32, 2), (3, 3), (9, 3), (48, 3),
                                   (4, 4), (8, 8), (32, 32)])
def test_what_is_planned_has_room(heads):
    """One group of up to 200 entries behind lists of every length: more parts than the workspace holds would be written past it."""
    hq, hkv = heads
    for n in range(1, 201):
        for pages in LENGTHS:
            for tokens in (1, 2) if n % 7 == 0 else (1,):
                fits(plan(hq, hkv, n, pages, tokens))


@pytest.mark.parametrize("hq,hkv,n,pages", [(1, 1, 129, 32000), (1, 1, 171, 6000), (1, 1, 176, 5692), (3, 3, 43, 32000), (2, 2, 43, 9200),
                                            (2, 1, 86, 9200)])
def test_few_rows_behind_long_lists(hq, hkv, n, pages):
    """Blocks of one entry each would be up to 176 of them, in parts for which the room was counted by blocks of 32 columns."""
    assert fits(plan(hq, hkv, n, pages)) == 32


@pytest.mark.parametrize("seed", range(8))
def test_groups_of_any_size(seed):
    rng = random.Random(seed)
    for _ in range(150):
        hkv = rng.choice([1, 1, 2, 3, 4, 6, 8])
        hq = hkv * rng.choice([1, 1, 2, 3, 6, 16])
        tokens, n = rng.choice([1, 1, 2, 3, 24]), rng.choice([1, 2, 5, 48, 130, 300])
        most = rng.choice([65, 130, 1025, 6000, 32768])
        group, common, pos = [], [], []
        while len(pos) < n:
            k, pages = min(rng.randint(1, 200), n - len(pos)), rng.randint(0, most - 2)
            for _ in range(k):
                far = min((pages + rng.choice([0, 1, 3])) * PAGE + rng.randrange(PAGE), most * PAGE - tokens)
                group.append(len(common)), pos.append(far if rng.random() < 0.95 else -1)
            common += [pages] * k
            group[-k:] = [len(common)] * k
        for g in (None, group):
            fits(V.vlac_plan_attention(pool(hkv, most), tokens, hq, pos, g, common if g else [0] * n))


def test_rules():
    # no long lists in the table: one block of 16 columns to a wave, as few entries to a block as one round of 256 items has room for
    # (600 entries of 6 columns: 225 blocks of 16 are a round, 600 of one entry and 300 of two are more)
    assert plan(6, 1, 8, 9)[0] == 6 and plan(6, 1, 600, 9)[0] == 16
    # 32 kv heads x 16 entries: 512 blocks of one entry are more than a round, 256 of two are one
    assert plan(32, 32, 16, 9)[0] == 2
    # one block for each of 32 heads over 1025 pages: 8 parts of it make a round of 256 items
    cols, (items, _), (parts, room) = plan(32, 32, 8, 1025)
    assert cols == 32 and parts == items == 256 and room == 2048
    # lists of up to 64 pages are left whole
    cols, (items, _), (parts, _) = plan(32, 32, 8, 62, max_pages=80)
    assert parts == 0


def test_refusals():
    out = [C.c_int() for _ in range(5)]
    refs = [C.byref(x) for x in out]
    lib, p = V.lib(), pool(2, 100)
    one = (C.c_int32 * 1)(40)
    call = lambda *a: lib.vlac_plan_attention(*a)
    assert call(C.byref(p), 1, 1, 4, one, None, one, *refs) == 0
    assert call(None, 1, 1, 4, one, None, one, *refs) == -1
    assert call(C.byref(p), 1, 1, 4, None, None, one, *refs) == -1 and call(C.byref(p), 1, 1, 4, one, None, None, *refs) == -1
    for k in range(5):
        assert call(C.byref(p), 1, 1, 4, one, None, one, *[None if i == k else r for i, r in enumerate(refs)]) == -1
    for n, tokens, hq, want in ((0, 1, 4, -3), (-1, 1, 4, -3), (4097, 1, 4, -3), (1, 0, 4, -3), (1, 65537, 4, -3), (1, 1, 0, -3), (1, 1, 3, -2),
                                (1, 1, 1026, -3)):
        assert call(C.byref(p), n, tokens, hq, one, None, one, *refs) == want, (n, tokens, hq)
    assert call(C.byref(p), 1, 100 * PAGE - 39, 4, one, None, one, *refs) == -3   # (beyond the table)
    assert call(C.byref(pool(0, 100)), 1, 1, 4, one, None, one, *refs) == -3
    with pytest.raises(ValueError):
        V.vlac_plan_attention(p, 1, 4, [40], None, [1, 1])
