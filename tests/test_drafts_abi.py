"""Drafted tokens, without a GPU: sizes, refusals before anything is queued, the binding's checks, and the plain model of trees that
the GPU tests compare with."""
import ctypes as C
import math

import pytest

import drafts_model as M
import paper_2502_02175_amd as V
from pages_model import E_RANGE as MODEL_RANGE, OK, Pool
from test_pages_abi import BAD_POINTERS, BAD_SIZES, E_NULL, E_RANGE, E_SHAPE, FAKE, pool

INF, NAN = math.inf, math.nan


def rot(**kw):
    f = dict(dims=64, layout=0, amplitude=1.0, turns=FAKE)
    f.update(kw)
    return V.Rotary(f["dims"], f["layout"], f["amplitude"], f["turns"])


def rules(**kw):
    r = V.TokenRules(1.0, 0.0, 0.0)
    r.tokens = 1
    for k, v in kw.items():
        setattr(r, k, v)
    return r


def calls(p, **kw):
    """Every call on a pool, one argument of which may be replaced."""
    f = dict(seqs=FAKE, pos=FAKE, n=3, tokens=2, layer=1, rot=rot(), places=None, hq=4, q=FAKE, q_stride=256, k=FAKE, v=FAKE, kv_stride=256,
             q_out=FAKE + 16, o_stride=256, q_gain=FAKE, k_gain=FAKE, eps=1e-6, group=None, parents=FAKE, out_places=None, ws=FAKE,
             ws_bytes=1 << 30, out=FAKE, path=FAKE, count=FAKE)
    f.update(kw)
    L, r = V.lib(), C.byref(p) if p is not None else None
    rt = C.byref(f["rot"]) if f["rot"] is not None else None
    return {
        "append": lambda: L.vlac_pages_append_rotated(r, f["layer"], f["seqs"], f["pos"], f["n"], f["tokens"], rt, f["places"], f["hq"],
                                                      f["q"], f["q_stride"], f["k"], f["v"], f["kv_stride"], f["q_out"], f["o_stride"],
                                                      f["q_gain"], f["k_gain"], f["eps"], None),
        "plan": lambda: L.vlac_attend_tree_plan(r, f["seqs"], f["pos"], f["n"], f["tokens"], f["hq"], f["group"], f["parents"],
                                                f["out_places"], f["ws"], f["ws_bytes"], None),
        "attend": lambda: L.vlac_attend_tree(r, f["layer"], f["n"], f["tokens"], f["hq"], f["q"], f["q_stride"], f["out"], f["ws"],
                                             f["ws_bytes"], None),
        "keep": lambda: L.vlac_pages_keep(r, f["seqs"], f["pos"], f["n"], f["tokens"], f["path"], f["count"], None),
    }


@pytest.mark.parametrize("kw,want", BAD_SIZES + BAD_POINTERS)
def test_every_call_refuses_a_pool_that_cannot_be(kw, want):
    for name, call in calls(pool(**kw)).items():
        assert call() == want, name


def test_every_call_refuses_no_pool():
    for name, call in calls(None).items():
        assert call() == E_NULL, name
    assert V.lib().vlac_decode_guided(None, C.byref(pool()), FAKE, 1, 1, None, 1, FAKE, C.byref(rules()), FAKE, None, FAKE, 1 << 30,
                                      None) == E_NULL
    assert V.lib().vlac_guided_workspace_bytes(None, C.byref(pool()), 1) == 0


@pytest.mark.parametrize("kw,names,want", [
    (dict(n=-1), "append plan attend keep", E_RANGE), (dict(n=4097), "append plan attend keep", E_RANGE),
    (dict(tokens=0), "append plan attend keep", E_RANGE), (dict(tokens=513), "plan attend keep", E_RANGE),
    (dict(tokens=(1 << 20) + 1), "append plan attend keep", E_RANGE), (dict(n=4096, tokens=257), "append plan attend", E_RANGE),
    (dict(layer=-1), "append attend", E_RANGE), (dict(layer=2), "append attend", E_RANGE),
    (dict(seqs=None), "append plan keep", E_NULL), (dict(pos=None), "append plan keep", E_NULL),
    (dict(k=None), "append", E_NULL), (dict(v=None), "append", E_NULL), (dict(q=None), "append attend", E_NULL),
    (dict(q_out=None), "append", E_NULL), (dict(out=None), "attend", E_NULL), (dict(parents=None), "plan", E_NULL),
    (dict(path=None), "keep", E_NULL), (dict(count=None), "keep", E_NULL),
    (dict(ws=None), "plan attend", E_NULL), (dict(ws=FAKE + 4), "plan attend", E_SHAPE), (dict(ws_bytes=1000), "plan attend", E_RANGE),
    (dict(kv_stride=248), "append", E_SHAPE), (dict(kv_stride=260), "append", E_SHAPE), (dict(kv_stride=-256), "append", E_SHAPE),
    (dict(q_stride=248), "append attend", E_SHAPE), (dict(q_stride=257), "append attend", E_SHAPE),
    (dict(q_stride=-256), "append attend", E_SHAPE), (dict(o_stride=248), "append", E_SHAPE), (dict(o_stride=260), "append", E_SHAPE),
    (dict(q_out=FAKE, o_stride=264), "append", E_SHAPE),               # in place with another stride
    (dict(q=FAKE + 2), "append attend", E_SHAPE), (dict(k=FAKE + 8), "append", E_SHAPE), (dict(v=FAKE + 2), "append", E_SHAPE),
    (dict(q_out=FAKE + 8), "append", E_SHAPE), (dict(q_gain=FAKE + 8), "append", E_SHAPE), (dict(k_gain=FAKE + 2), "append", E_SHAPE),
    (dict(out=FAKE + 2), "attend", E_SHAPE), (dict(hq=1025), "append", E_RANGE), (dict(hq=-1), "append", E_RANGE),
    (dict(hq=6), "plan attend", E_SHAPE), (dict(hq=0), "plan attend", E_RANGE),
    (dict(eps=-1e-6), "append", E_RANGE), (dict(eps=NAN), "append", E_RANGE), (dict(eps=INF), "append", E_RANGE),
    (dict(rot=rot(dims=0)), "append", E_SHAPE), (dict(rot=rot(dims=3)), "append", E_SHAPE), (dict(rot=rot(dims=66)), "append", E_SHAPE),
    (dict(rot=rot(layout=2)), "append", E_RANGE), (dict(rot=rot(layout=-1)), "append", E_RANGE),
    (dict(rot=rot(amplitude=NAN)), "append", E_RANGE), (dict(rot=rot(turns=None)), "append", E_NULL),
    (dict(rot=rot(turns=FAKE + 4)), "append", E_SHAPE),
    (dict(n=0), "append plan attend keep", 0),
    (dict(n=0, hq=0, q=None, q_out=None, q_stride=0, o_stride=0, rot=None, q_gain=None, k_gain=None, eps=NAN), "append", 0),
])
def test_arguments_that_are_refused_on_the_host(kw, names, want):
    all_calls = calls(pool(), **kw)
    for name in names.split():
        assert all_calls[name]() == want, name


def test_tree_workspace():
    p = pool(max_pages=80)
    for T in (1, 2, 33, 512):
        rows = 5 * T * ((T + 62) // 32 + 1) * 4
        a, b = V.vlac_attend_workspace_bytes(p, 5, T, 4), V.vlac_attend_tree_workspace_bytes(p, 5, T, 4)
        assert a + rows <= b < a + rows + 256
    assert V.vlac_attend_tree_workspace_bytes(p, 0, 3, 4) > 0
    for n, t, h in ((-1, 1, 4), (4097, 1, 4), (4, 0, 4), (4, 513, 4), (4, 1, 6), (4, 1, 0)):
        assert V.vlac_attend_tree_workspace_bytes(p, n, t, h) == 0
    assert V.vlac_attend_tree_workspace_bytes(None, 1, 1, 4) == 0


@pytest.mark.parametrize("kw,want", [
    (dict(dims=0), E_SHAPE), (dict(dims=130), E_SHAPE), (dict(dims=31), E_SHAPE), (dict(base=1.0), E_RANGE), (dict(base=NAN), E_RANGE),
    (dict(base=INF), E_RANGE), (dict(factor=0.5), E_RANGE), (dict(original=-1.0), E_RANGE), (dict(original=INF), E_RANGE),
    (dict(low=-1.0), E_RANGE), (dict(low=4.0), E_RANGE), (dict(high=NAN), E_RANGE), (dict(turns=None), E_NULL),
    (dict(turns=FAKE + 4), E_SHAPE)])
def test_rotary_tables_that_are_refused(kw, want):
    f = dict(dims=64, base=1e4, factor=2.0, original=4096.0, low=1.0, high=4.0, turns=FAKE)
    f.update(kw)
    assert V.lib().vlac_rotary_fill(*f.values(), None) == want


def choose(r, **kw):
    f = dict(logits=FAKE, rows=4, vocab=100, stride=100, out=FAKE, out_stride=100, token=FAKE, ws=FAKE, ws_bytes=1 << 20)
    f.update(kw)
    return V.lib().vlac_choose_tokens(f["logits"], f["rows"], f["vocab"], f["stride"], C.byref(r) if r is not None else None, f["out"],
                                      f["out_stride"], f["token"], f["ws"], f["ws_bytes"], None)


@pytest.mark.parametrize("kw,want", [
    (dict(rows=-1), E_RANGE), (dict(rows=(1 << 20) + 1), E_RANGE), (dict(vocab=0), E_RANGE), (dict(vocab=(1 << 24) + 1), E_RANGE),
    (dict(stride=99), E_SHAPE), (dict(out_stride=99), E_SHAPE), (dict(out_stride=101), E_SHAPE), (dict(stride=-100), E_SHAPE),
    (dict(logits=None), E_NULL), (dict(ws=None), E_NULL), (dict(ws=FAKE + 8), E_SHAPE), (dict(ws_bytes=8), E_RANGE),
    (dict(logits=FAKE + 2, out=FAKE + 402), E_SHAPE), (dict(out=FAKE + 2), E_SHAPE), (dict(token=FAKE + 1), E_SHAPE),
    (dict(rows=0), 0), (dict(out=None, token=None, ws=None), 0)])
def test_choices_that_are_refused(kw, want):
    assert choose(rules(), **kw) == want


@pytest.mark.parametrize("kw,want", [
    (dict(repetition=0.0), E_RANGE), (dict(repetition=-1.0), E_RANGE), (dict(repetition=NAN), E_RANGE), (dict(repetition=INF), E_RANGE),
    (dict(presence=NAN), E_RANGE), (dict(frequency=INF), E_RANGE), (dict(tokens=0), E_RANGE), (dict(tokens=513), E_RANGE),
    (dict(history=FAKE), E_NULL), (dict(history_len=FAKE), E_NULL), (dict(parents=FAKE), E_NULL), (dict(drafted=FAKE), E_NULL),
    (dict(tokens=2), E_NULL), (dict(tokens=3, parents=FAKE, drafted=FAKE), E_SHAPE),
    (dict(bias=FAKE, bias_stride=99), E_SHAPE), (dict(bias=FAKE, bias_stride=-1), E_SHAPE), (dict(allowed=FAKE, allowed_stride=3), E_SHAPE),
    (dict(history=FAKE, history_len=FAKE, history_stride=-1), E_SHAPE), (dict(bias=FAKE + 2), E_SHAPE), (dict(allowed=FAKE + 1), E_SHAPE)])
def test_rules_that_are_refused(kw, want):
    assert choose(rules(**kw)) == want
    assert choose(None) == E_NULL


def test_choose_workspace():
    assert V.vlac_choose_workspace_bytes(0, 1) > 0
    assert V.vlac_choose_workspace_bytes(300, 100003) >= 300 * 8 * (100003 // 65536)
    for rows, vocab in ((-1, 5), ((1 << 20) + 1, 5), (1, 0), (1, (1 << 24) + 1)):
        assert V.vlac_choose_workspace_bytes(rows, vocab) == 0


def accept(**kw):
    f = dict(parents=FAKE, drafted=FAKE, chosen=FAKE, n=2, tokens=5, path=FAKE, count=FAKE, token=FAKE)
    f.update(kw)
    return V.lib().vlac_tree_accept(*f.values(), None)


@pytest.mark.parametrize("kw,want", [
    (dict(n=-1), E_RANGE), (dict(n=4097), E_RANGE), (dict(tokens=0), E_RANGE), (dict(tokens=513), E_RANGE), (dict(n=0), 0)] + [
    (dict([(k, None)]), E_NULL) for k in ("parents", "drafted", "chosen", "path", "count", "token")])
def test_accepting_that_is_refused(kw, want):
    assert accept(**kw) == want


def test_binding_refuses_what_does_not_fit():
    import torch
    x, f = torch.zeros((4, 5), dtype=torch.int32), torch.zeros((4, 100))
    with pytest.raises(ValueError):
        V.rotary(64, turns=torch.zeros(32, dtype=torch.float64))
    with pytest.raises(ValueError):
        V.vlac_choose_tokens(f, rules(), f, None, None)
    with pytest.raises(ValueError):
        V.token_rules(bias=torch.zeros(100))
    with pytest.raises(ValueError):
        V.token_rules(history=x)
    with pytest.raises(ValueError):
        V.token_rules(drafted=x)
    with pytest.raises(ValueError):
        V.vlac_tree_accept(x, x, x, 4, 5, x, x, x)
    with pytest.raises(ValueError):
        V.vlac_pages_keep(pool(), x[0], x[0], 4, 5, x, x[0])
    h = torch.zeros((1, 2, 4, 64), dtype=torch.float16)
    with pytest.raises(ValueError):
        V.vlac_pages_append_rotated(pool(), 0, FAKE, FAKE, 1, 2, None, None, 4, h, FAKE, FAKE, FAKE)
    assert V.vlac_pages_keep(pool(), FAKE, FAKE, -1, 5, FAKE, FAKE, check=False) == E_RANGE
    assert V.vlac_tree_accept(FAKE, FAKE, FAKE, 0, 5, FAKE, FAKE, FAKE) == 0
    with pytest.raises(V.VlacError):
        V.vlac_attend_tree_plan(pool(), FAKE, FAKE, 1, 600, 4, None, FAKE, None, None)


# ---- the model itself, by hand ----

def test_model_of_trees():
    par = [-1, 0, 0, 1, -1, 3, -2, 6, 9]
    assert M.lineage(par, 5) == [5, 3, 1, 0] and M.lineage(par, 4) == [4]
    assert M.lineage(par, 6) is None and M.lineage(par, 7) is None and M.lineage(par, 8) is None
    assert M.places(par, 10) == [10, 11, 11, 12, 10, 13, -1, -1, -1]
    assert M.accept(par, [7, 3, 4, 9, 7, 1, 0, 0, 0], [4, 0, 8, 0, 0, 0, 0, 0, 0]) == ([0, 2], 8)
    assert M.accept([-2, 0], [1, 1], [1, 1]) == ([], -1)


def test_model_of_keeping():
    p = Pool(8, 3, 3)
    assert p.extend([0, 1], 60) == [0, 0] and p.extend([0, 1], 10) == [60, 60]
    assert p.table[0] == [0, 1, 4] and p.table[1] == [2, 3, 5]
    moves = M.keep(p, [0, 1, 0], [60, 60, 60], 10, [[0, 3, 9], [0], [0]], [3, 1, 1])
    assert moves == [(0, 63, 61), (0, 69, 62)] and p.len == [63, 61, 0] and p.table[0] == [0, 1, -1] and p.refs == [1, 1, 1, 1, 0, 0, 0, 0]
    assert p.check() == MODEL_RANGE
    assert p.extend([0], 2) == [63] and M.keep(p, [0, -1], [63, -1], 2, [[0, 1], [0, 0]], [2, 5]) == [] and p.check() == OK and p.len[0] == 65
