"""The cases of test_gpu_attend once more in pools with longer tables: with room for more than 64 pages per sequence a list may be cut
into parts, and another kernel (blocks of 32 columns) does what the short tables leave to the one for 16; with many more entries
than columns fit in a round of the chip neither cuts."""
import pytest

import paper_2502_02175_amd as V
import test_gpu_attend as T

pytestmark = pytest.mark.gpu


@pytest.fixture
def long_tables(monkeypatch):
    short = V.new_pages

    def new_pages(n_layers, n_kv_heads, head_dim, operand, n_pages, max_seqs, max_pages, device="cuda"):
        return short(n_layers, n_kv_heads, head_dim, operand, n_pages, max_seqs, max(max_pages, 70), device)

    monkeypatch.setattr(V, "new_pages", new_pages)


@pytest.mark.parametrize("hq,hkv,hd", [(4, 4, 64), (12, 2, 128), (8, 1, 128), (6, 3, 64)])
@pytest.mark.parametrize("operand", [0, 1])
@pytest.mark.parametrize("tokens", [1, 5])
def test_groups_of_several_prefixes(long_tables, hq, hkv, hd, operand, tokens):
    T.test_groups_of_several_prefixes(hq, hkv, hd, operand, tokens)


@pytest.mark.parametrize("length", [1, 32, 33, 64, 700])
@pytest.mark.parametrize("hq,hkv,hd,operand", [(4, 4, 64, 1), (12, 2, 128, 0)])
def test_one_sequence_of_any_length(long_tables, length, hq, hkv, hd, operand):
    T.test_one_sequence_of_any_length(length, hq, hkv, hd, operand)


@pytest.mark.parametrize("operand", [0, 1])
def test_values_at_the_ends_of_the_type(long_tables, operand):
    T.test_values_at_the_ends_of_the_type(operand)


@pytest.mark.parametrize("name", ["test_groups_are_a_hint", "test_entries_that_do_not_fit_get_zeros",
                                  "test_nan_and_infinity_stay_where_they_are_seen",
                                  "test_layers_strided_queries_and_what_lies_around", "test_own_parts_behind_a_short_stem",
                                  "test_a_plan_serves_every_layer_and_another_stream", "test_a_workspace_without_its_plan_is_not_used"])
def test_the_others(long_tables, name):
    getattr(T, name)()


@pytest.mark.parametrize("hq,hkv,hd,operand", [(32, 32, 64, 1), (16, 8, 128, 0)])
@pytest.mark.parametrize("n,tokens", [(1, 1), (5, 3), (127, 1), (128, 1), (129, 1), (140, 2)])
def test_around_one_round_of_the_chip(hq, hkv, hd, operand, n, tokens):
    """Short tables: as many columns as blocks of 16 fill the chip once, and a few more or less."""
    c = T.Cache(hkv, hd, operand, seed=n)
    stems = [[c._new(T.PAGE) for _ in range(k)] for k in (0, 3, 9)]
    pos = [32 * (0, 3, 9)[i % 3] + (5 * i) % 70 for i in range(n)]
    order = sorted(range(n), key=lambda i: i % 3)
    seqs = [c.sequence(pos[i] + tokens, stems[i % 3]) for i in order]
    T.compare(c, c.pool(), seqs, [pos[i] for i in order], T.queries(c, n, tokens, hq), [i % 3 for i in order])


@pytest.mark.parametrize("hq,hkv,hd,operand", [(4, 4, 64, 1), (12, 2, 128, 0)])
@pytest.mark.parametrize("stem", [3, 90])
def test_far_values_in_a_place_that_some_rows_see(hq, hkv, hd, operand, stem):
    """An infinite and a NaN value of V at the second of three new tokens: the first row does not see it, the others' features
    are what it makes of them; over a short list, and over one that is cut into parts."""
    import torch
    c = T.Cache(hkv, hd, operand, seed=stem)
    base = [c._new(T.PAGE) for _ in range(stem)]
    pos = [32 * stem + 4 + i for i in range(5)]
    seqs = [c.sequence(x + 3, base) for x in pos]
    at = pos[1] + 1
    page = c.pages[c.seqs[seqs[1]][0][at // 32]]
    page[0, 1, at % 32, 0, 5] = float("inf")
    page[0, 1, at % 32, hkv - 1, 6] = float("nan")
    q = T.queries(c, 5, 3, hq)
    got = T.run(c.pool(), c, seqs, pos, q, [0] * 5).double()
    g = hq // hkv
    for i in range(5):
        for t in range(3):
            want, tol = T.definition(c, [seqs[i]], [pos[i] + t], q[i:i + 1, t:t + 1])
            if i == 1 and t > 0:
                assert bool((got[i, t, :g, 5] == float("inf")).all()) and bool(got[i, t, hq - g:, 6].isnan().all())
            fine = want[0, 0].isfinite()
            assert fine.sum() == hq * hd - (2 * g if i == 1 and t > 0 else 0)
            assert bool(((got[i, t] - want[0, 0]).abs() <= tol[0, 0])[fine].all()), (i, t)
