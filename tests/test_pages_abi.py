"""Pages of the cache and attention over them, without a GPU: sizes, refusals before anything is queued, and the plain
model of the pool that the GPU tests compare with."""
import ctypes as C

import pytest

import paper_2502_02175_amd as V
from pages_model import OK, E_NOMEM, E_RANGE as MODEL_RANGE, PAGE, Pool, k_tile_at, v_tile_at

E_NULL, E_SHAPE, E_RANGE = -1, -2, -3
FAKE = 1 << 20   # an aligned address that no refused call looks at


def pool(**kw):
    f = dict(n_layers=2, n_kv_heads=4, head_dim=64, operand_dtype=1, n_pages=16, max_seqs=8, max_pages=4, data=FAKE,
             refs=FAKE, table=FAKE, len=FAKE, scratch=FAKE)
    f.update(kw)
    return V.Pages(**f)


def test_sizes():
    assert V.vlac_page_bytes(pool()) == 2 * 2 * 4 * 32 * 64 * 2
    assert V.vlac_pages_scratch_bytes(pool()) >= 4 * (3 * 16 + 2 * 8)
    assert V.vlac_page_bytes(pool(data=None, refs=None)) > 0          # (the pointers are not looked at)
    for kw in BAD_SIZES:
        assert V.vlac_page_bytes(pool(**kw[0])) == 0 and V.vlac_pages_scratch_bytes(pool(**kw[0])) == 0
        assert V.vlac_attend_workspace_bytes(pool(**kw[0]), 4, 1, 4) == 0
    assert V.vlac_attend_workspace_bytes(pool(), 4, 1, 4) > 0
    assert V.vlac_attend_workspace_bytes(pool(), 0, 1, 4) > 0
    for n, t, h in ((-1, 1, 4), (4097, 1, 4), (4, 0, 4), (4, 65537, 4), (17, 65536, 4), (4, 1, 6), (4, 1, 2), (4, 1, 0), (4, 1, 1028)):
        assert V.vlac_attend_workspace_bytes(pool(), n, t, h) == 0
    assert V.vlac_page_bytes(None) == 0 and V.vlac_attend_workspace_bytes(None, 1, 1, 4) == 0
    # parts are bounded: a batch that fills the chip by itself is not cut into many
    rows = 1024 * 1024
    assert V.vlac_attend_workspace_bytes(pool(), 1024, 256, 4) < 2.2 * rows * (64 + 2) * 4 + (1 << 22)


BAD_SIZES = [(dict(n_layers=0), E_RANGE), (dict(n_layers=513), E_RANGE), (dict(n_kv_heads=0), E_RANGE), (dict(n_pages=0), E_RANGE),
             (dict(n_pages=(1 << 24) + 1), E_RANGE), (dict(max_seqs=0), E_RANGE), (dict(max_seqs=65537), E_RANGE),
             (dict(max_pages=0), E_RANGE), (dict(max_pages=32769), E_RANGE), (dict(head_dim=96), E_SHAPE),
             (dict(operand_dtype=3), E_RANGE), (dict(operand_dtype=-1), E_RANGE)]
BAD_POINTERS = [(dict(data=None), E_NULL), (dict(refs=None), E_NULL), (dict(table=None), E_NULL), (dict(len=None), E_NULL),
                (dict(scratch=None), E_NULL), (dict(data=FAKE + 8), E_SHAPE)]


def calls(p, **kw):
    """Every call on the pool `p`, one argument of which may be replaced."""
    f = dict(src=FAKE, dst=FAKE, seqs=FAKE, pos=FAKE, n=3, tokens=2, layer=1, k=FAKE, v=FAKE, stride=256, live=FAKE, hq=4, q=FAKE,
             q_stride=256, out=FAKE, ws=FAKE, group=None, ws_bytes=1 << 30)
    f.update(kw)
    L, r = V.lib(), C.byref(p) if p is not None else None
    return {
        "fork": lambda: L.vlac_pages_fork(r, f["src"], f["dst"], f["n"], 0, None),
        "extend": lambda: L.vlac_pages_extend(r, f["seqs"], f["n"], f["tokens"], f["pos"], None),
        "append": lambda: L.vlac_pages_append(r, f["layer"], f["seqs"], f["pos"], f["n"], f["tokens"], f["k"], f["v"], f["stride"], None),
        "free": lambda: L.vlac_pages_free(r, f["seqs"], f["n"], None),
        "compact": lambda: L.vlac_pages_compact(r, f["live"], None),
        "plan": lambda: L.vlac_attend_plan(r, f["seqs"], f["pos"], f["n"], f["tokens"], f["hq"], f["group"], f["ws"], f["ws_bytes"], None),
        "attend": lambda: L.vlac_attend_shared(r, f["layer"], f["n"], f["tokens"], f["hq"], f["q"], f["q_stride"], f["out"], f["ws"],
                                               f["ws_bytes"], None),
        "reset": lambda: L.vlac_pages_reset(r, None),
        "check": lambda: L.vlac_pages_check(r, None),
    }


@pytest.mark.parametrize("kw,want", BAD_SIZES + BAD_POINTERS)
def test_every_call_refuses_a_pool_that_cannot_be(kw, want):
    for name, call in calls(pool(**kw)).items():
        assert call() == want, name


def test_every_call_refuses_no_pool():
    for name, call in calls(None).items():
        assert call() == E_NULL, name
    assert V.lib().vlac_pages_import(None, FAKE, 1, 1, C.byref(pool()), FAKE, None) == E_NULL
    assert V.lib().vlac_decode_candidates(None, C.byref(pool()), FAKE, 1, 1, None, 1, FAKE, FAKE, None, FAKE, 1 << 30, None) == E_NULL
    assert V.lib().vlac_candidates_workspace_bytes(None, C.byref(pool()), 1) == 0


@pytest.mark.parametrize("kw,names,want", [
    (dict(n=-1), "fork extend append free plan attend", E_RANGE), (dict(n=4097), "fork extend append free plan attend", E_RANGE),
    (dict(tokens=0), "extend append plan attend", E_RANGE), (dict(tokens=-3), "extend append plan attend", E_RANGE),
    (dict(tokens=(1 << 20) + 1), "extend append plan attend", E_RANGE),
    (dict(layer=-1), "append attend", E_RANGE), (dict(layer=2), "append attend", E_RANGE),
    (dict(src=None), "fork", E_NULL), (dict(dst=None), "fork", E_NULL), (dict(seqs=None), "extend append free plan", E_NULL),
    (dict(pos=None), "extend append plan", E_NULL), (dict(k=None), "append", E_NULL), (dict(v=None), "append", E_NULL),
    (dict(live=None), "compact", E_NULL), (dict(q=None), "attend", E_NULL), (dict(out=None), "attend", E_NULL),
    (dict(ws=None), "plan attend", E_NULL), (dict(ws=FAKE + 4), "plan attend", E_SHAPE), (dict(ws_bytes=1000), "plan attend", E_RANGE),
    (dict(stride=248), "append", E_SHAPE), (dict(stride=260), "append", E_SHAPE), (dict(stride=0), "append", E_SHAPE),
    (dict(stride=-256), "append", E_SHAPE), (dict(k=FAKE + 2), "append", E_SHAPE), (dict(v=FAKE + 8), "append", E_SHAPE),
    (dict(q_stride=248), "attend", E_SHAPE), (dict(q_stride=-256), "attend", E_SHAPE), (dict(q_stride=257), "attend", E_SHAPE),
    (dict(q=FAKE + 2), "attend", E_SHAPE), (dict(out=FAKE + 2), "attend", E_SHAPE),
    (dict(hq=6), "plan attend", E_SHAPE), (dict(hq=0), "plan attend", E_RANGE), (dict(hq=1028), "plan attend", E_RANGE),
    (dict(n=0), "fork extend append free plan attend", 0),
])
def test_arguments_that_are_refused_on_the_host(kw, names, want):
    all_calls = calls(pool(), **kw)
    for name in names.split():
        assert all_calls[name]() == want, name


def test_binding_refuses_host_tensors():
    import torch
    with pytest.raises(ValueError):
        V.pages(2, 4, 64, 1, torch.zeros(16 * 65536, dtype=torch.uint8), torch.zeros(16, dtype=torch.int32),
                torch.zeros((8, 4), dtype=torch.int32), torch.zeros(8, dtype=torch.int32))
    with pytest.raises(V.VlacError):
        V.pages(2, 4, 96, 1, torch.zeros(16), torch.zeros(16, dtype=torch.int32), torch.zeros((8, 4), dtype=torch.int32),
                torch.zeros(8, dtype=torch.int32))


# ---- the model itself, by hand ----

def test_model_fork_shares_full_pages_and_copies_the_last():
    p = Pool(8, 4, 4)
    assert p.extend([2], 70) == [0] and p.table[2] == [0, 1, 2, -1] and p.len[2] == 70
    p.fork([2, 2], [0, 3])
    assert p.table[0] == [0, 1, 3, -1] and p.table[3] == [0, 1, 4, -1]
    assert p.refs == [3, 3, 1, 1, 1, 0, 0, 0] and p.data[3] == p.data[4] == 2
    p.fork([2], [0], deep=True)                       # page 3 comes back first
    assert p.table[0] == [3, 5, 6, -1] and p.refs == [2, 2, 1, 1, 1, 1, 1, 0]
    p.free([2, 2])
    assert p.refs == [1, 1, 0, 1, 1, 1, 1, 0] and p.check() == OK
    assert p.compact() == 6 and p.table[0] == [3, 5, 2, -1] and p.data[2] == 2
    p.fork([0, 0], [1, 2], deep=True)
    assert p.check() == E_NOMEM and p.len[1] == 0 and p.refs == [1, 1, 1, 1, 1, 1, 0, 0]
    p.fork([0, 3, 9], [0, 1, 2])
    assert p.check() == MODEL_RANGE and p.len[1] == 70 and p.len[2] == 0


def test_tile_orders_are_permutations():
    for hd in (64, 128):
        for at in (k_tile_at(hd), v_tile_at(hd)):
            assert sorted(at.ravel()) == list(range(PAGE * hd))
