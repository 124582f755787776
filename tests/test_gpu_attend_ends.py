"""Attention over V of the type's largest value: the result is an average, so it is no larger, whatever the weights round to.

The keys of a list are one of each page, at rising scores, and 31 others that all score 0: their weights are equal and round
the same way, so that the rounded weights sum to more than the unrounded ones in a good part of the columns, each of which has a
score distance of its own."""
import pytest

from test_gpu_attend import Cache, compare, definition, run
from test_gpu_attend import DEV
from test_gpu_attend_tables import long_tables  # noqa: F401

pytestmark = pytest.mark.gpu


def of_one_value(hkv, hd, operand, pages, T, hq, n, value, top=9.0):
    """-> cache, the one sequence, position, queries: column c's distance between the highest score and 0 is up to `top` in log2."""
    import torch
    c = Cache(hkv, hd, operand, seed=pages)
    length = 32 * pages - 3
    s = c.sequence(length)
    key = torch.zeros((hkv, hd), device=DEV, dtype=c.dt)
    key[:, 0] = 4.0
    for j, page in enumerate(c.seqs[s][0]):
        filled = min(32, length - 32 * j)
        c.pages[page][:, 0, :filled] = 0.0
        c.pages[page][:, 0, 5] = key * (0.5 + 0.5 * (j + 1) / pages)
        c.pages[page][:, 1, :filled] = value
    q = torch.zeros((n, T, hq, hd), device=DEV, dtype=c.dt)
    q[..., 0] = torch.linspace(0.0, top * hd ** 0.5 / 4.0 / 1.4427, n * T * hq, device=DEV).view(n, T, hq).to(c.dt)
    return c, s, length - T, q


TYPES = [0, 1]
CASES = [(8, 1, 64, 60, 1), (8, 8, 64, 30, 1), (12, 2, 128, 30, 3)]


def largest(operand):
    import torch
    return torch.finfo(torch.bfloat16 if operand == 0 else torch.float16).max


def check(hq, hkv, hd, n, T, pages, operand, sign):
    c, s, pos, q = of_one_value(hkv, hd, operand, pages, T, hq, n, sign * largest(operand))
    compare(c, c.pool(), [s] * n, [pos] * n, q)


@pytest.mark.parametrize("sign", [1, -1])
@pytest.mark.parametrize("operand", TYPES)
@pytest.mark.parametrize("pages", [1, 2, 9, 20])
@pytest.mark.parametrize("hq,hkv,hd,n,T", CASES)
def test_averages_of_the_largest_value(hq, hkv, hd, n, T, pages, operand, sign):
    check(hq, hkv, hd, n, T, pages, operand, sign)


@pytest.mark.parametrize("sign", [1, -1])
@pytest.mark.parametrize("operand", TYPES)
@pytest.mark.parametrize("pages", [1, 9, 80, 300])
@pytest.mark.parametrize("hq,hkv,hd,n,T", CASES)
def test_averages_of_the_largest_value_in_long_tables(long_tables, hq, hkv, hd, n, T, pages, operand, sign):  # noqa: F811
    """(blocks of 32 columns; the lists of 80 and 300 pages in parts)"""
    check(hq, hkv, hd, n, T, pages, operand, sign)


@pytest.mark.parametrize("operand", TYPES)
@pytest.mark.parametrize("pages", [3, 80])
def test_what_is_infinite_stays_infinite(operand, pages):
    """One infinite value among the largest ones, and one NaN: of two features each."""
    import torch
    hq, hkv, hd, n = 8, 2, 64, 20
    c, s, pos, q = of_one_value(hkv, hd, operand, pages, 1, hq, n, largest(operand), top=5.0)
    page = c.pages[c.seqs[s][0][pages // 2]]
    page[0, 1, 7, :, 1] = float("inf")
    page[0, 1, 9, :, 2] = -float("inf")
    page[0, 1, 11, :, 3] = float("nan")
    out = run(c.pool(), c, [s] * n, [pos] * n, q)
    want, tol = definition(c, [s] * n, [pos] * n, q)
    assert bool((out[..., 1] == float("inf")).all()) and bool((out[..., 2] == -float("inf")).all())
    assert bool(torch.isnan(out[..., 3]).all())
    fine = [0] + list(range(4, hd))
    assert bool(((out.double() - want).abs() <= tol)[..., fine].all())
