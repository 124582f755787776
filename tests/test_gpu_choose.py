"""The choice of tokens under rules against numpy's fp32, whose every operation is rounded as the rules say: bit for bit."""
import math
import random

import numpy as np
import pytest

import drafts_model as M
import paper_2502_02175_amd as V

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F = np.float32


def gpu(x, dtype=None):
    import torch
    return torch.tensor(np.asarray(x), device=DEV, dtype=dtype)


def apply(logits, texts, repetition=1.0, presence=0.0, frequency=0.0, bias=None, allowed=None):
    """logits [rows, vocab] fp32; texts: the tokens of every row; bias [rows or 1, vocab]; allowed bools the same."""
    x = np.array(logits, dtype=F)
    vocab = x.shape[1]
    with np.errstate(all="ignore"):
        for r, text in enumerate(texts):
            n = np.bincount([t for t in text if 0 <= t < vocab], minlength=vocab)
            hit = n > 0
            y = np.where(x[r] > 0, x[r] / F(repetition), x[r] * F(repetition)).astype(F)
            y = (y - F(presence)).astype(F)
            y = (y - (F(frequency) * n.astype(F)).astype(F)).astype(F)
            x[r] = np.where(hit, y, x[r])
        if bias is not None:
            x = (x + np.asarray(bias, dtype=F)).astype(F)
        if allowed is not None:
            x = np.where(allowed, x, F(-math.inf))
    y = np.where(np.isnan(x), F(-math.inf), x)
    token = np.where(y.max(1) > -math.inf, y.argmax(1), -1)
    return x, token.astype(np.int32)


def bits(allowed):
    """bools [.., vocab] -> int32 words."""
    a = np.asarray(allowed)
    a = np.concatenate([a, np.ones(a.shape[:-1] + (-a.shape[-1] % 32,), bool)], -1)
    w = (a.reshape(a.shape[:-1] + (-1, 32)).astype(np.uint64) << np.arange(32, dtype=np.uint64)).sum(-1)
    return w.astype(np.uint32).view(np.int32)


def same(a, b):
    return np.array_equal(np.asarray(a, F).view(np.int32)[~np.isnan(a)], np.asarray(b, F).view(np.int32)[~np.isnan(b)]) and \
        np.array_equal(np.isnan(a), np.isnan(b))


def check(logits, rules, want, token, stride=None):
    """Out of place, in place, and one of the two outputs alone."""
    import torch
    rows, vocab = logits.shape
    wide = torch.full((rows, stride or vocab), 5.0, device=DEV)
    wide[:, :vocab] = gpu(logits)
    x = wide[:, :vocab]
    ws = torch.empty(V.vlac_choose_workspace_bytes(rows, vocab), dtype=torch.uint8, device=DEV)
    ws.fill_(0xFF)
    out, tok = torch.full((rows, vocab), 7.0, device=DEV), torch.full((rows,), -7, dtype=torch.int32, device=DEV)
    V.vlac_choose_tokens(x, rules, out, tok, ws)
    assert same(out.cpu().numpy(), want) and tok.tolist() == token.tolist()
    assert same(x.cpu().numpy(), logits)
    tok.fill_(-7)
    V.vlac_choose_tokens(x, rules, None, tok, ws)
    assert tok.tolist() == token.tolist()
    V.vlac_choose_tokens(x, rules, x, None, None)
    assert same(x.cpu().numpy(), want) and bool((wide[:, vocab:] == 5).all())


VOCABS = [1, 2, 31, 32, 33, 100, 1023, 8191, 8192, 8193, 16385, 40001]


@pytest.mark.parametrize("vocab", VOCABS)
@pytest.mark.parametrize("rows", [1, 3, 70])
def test_everything_at_once(vocab, rows):
    rng = np.random.default_rng(vocab + rows)
    logits = (3 * rng.standard_normal((rows, vocab))).astype(F)
    most = 50
    history = (rng.random((rows, most)) ** 3 * (vocab + 5)).astype(np.int32) - 2          # some outside the vocabulary
    length = rng.integers(-2, most + 9, rows).astype(np.int32)                             # negative, and more than there is
    texts = [history[r, :min(max(length[r], 0), most)] for r in range(rows)]
    bias = np.where(rng.random((rows, vocab)) < 0.2, rng.standard_normal((rows, vocab)), 0).astype(F)
    allowed = rng.random((rows, vocab)) < 0.7
    price = dict(repetition=1.3, presence=0.4, frequency=0.25)
    want, token = apply(logits, texts, **price, bias=bias, allowed=allowed)
    r = V.token_rules(**price, bias=gpu(bias), allowed=gpu(bits(allowed)), history=gpu(history), history_len=gpu(length))
    check(logits, r, want, token, stride=vocab + 3)
    # one bias and one mask for all rows
    want, token = apply(logits, texts, **price, bias=bias[:1], allowed=allowed[:1])
    r = V.token_rules(**price, bias=gpu(bias[0]), allowed=gpu(bits(allowed[0])), history=gpu(history), history_len=gpu(length))
    check(logits, r, want, token)


@pytest.mark.parametrize("price", [dict(), dict(repetition=0.5), dict(repetition=1.7), dict(presence=1.5), dict(frequency=0.3),
                                   dict(presence=-0.5, frequency=-0.25)])
def test_each_rule_alone(price):
    rng = np.random.default_rng(3)
    rows, vocab, most = 5, 9001, 3000
    logits = (2 * rng.standard_normal((rows, vocab))).astype(F)
    logits[0, :40] = 0.0
    logits[1, :40] = -0.0
    history = (rng.random((rows, most)) ** 4 * vocab).astype(np.int32)
    length = np.array([most, 0, 1, 700, 2999], np.int32)
    texts = [history[r, :length[r]] for r in range(rows)]
    want, token = apply(logits, texts, **price)
    check(logits, V.token_rules(**price, history=gpu(history), history_len=gpu(length)), want, token)
    want, token = apply(logits, [[]] * rows, **price)
    check(logits, V.token_rules(**price), want, token)
    ban = np.zeros(vocab, F)
    ban[int(token[2])] = -math.inf
    want, token = apply(logits, [[]] * rows, bias=ban[None])
    check(logits, V.token_rules(bias=gpu(ban)), want, token)


def test_ties_nan_and_nothing_allowed():
    rng = np.random.default_rng(5)
    rows, vocab = 12, 20000
    x = rng.integers(-3, 4, (rows, vocab)).astype(F)             # ties everywhere: the lowest
    x[1, rng.integers(0, vocab, 50)] = math.nan
    x[2] = math.nan
    x[3] = -math.inf
    x[4, 777], x[4, 12345] = math.inf, math.inf
    x[5, :] = -math.inf
    x[5, vocab - 1] = -3e38
    x[6, :] = 2.5
    allowed = np.ones((rows, vocab), bool)
    allowed[0, :vocab // 2] = False
    allowed[7] = False                                           # nothing
    allowed[8] = False
    allowed[8, 8192] = True                                      # one, the first of a piece
    allowed[9] = False
    allowed[9, 8191] = True                                      # the last
    x[10, 5], allowed[10, 5] = math.nan, False                   # masked places: whatever they hold
    x[11, 6], allowed[11, 6] = math.inf, False
    text = [[t for t in (5, 6, 777, 777, 12345, vocab - 1)]] * rows
    for price in (dict(), dict(repetition=2.0, presence=0.5)):
        want, token = apply(x, text, **price, allowed=allowed)
        assert token[7] == -1 and token[2] == -1 and token[3] == -1 and token[8] == 8192 and token[9] == 8191
        r = V.token_rules(**price, allowed=gpu(bits(allowed)), history=gpu(np.array(text, np.int32)),
                          history_len=gpu(np.full(rows, 6, np.int32)))
        check(x, r, want, token)


@pytest.mark.parametrize("n,T,vocab", [(1, 2, 50), (3, 33, 8200), (2, 512, 300), (9, 7, 33000)])
@pytest.mark.parametrize("kind", ["random", "holes", "chain"])
def test_nodes_of_trees(n, T, vocab, kind):
    rng = np.random.default_rng(T)
    pr = random.Random(T)
    rows = n * T
    logits = (3 * rng.standard_normal((rows, vocab))).astype(F)
    trees = [M.tree(pr, T, kind, pr.randint(1, T)) for _ in range(n)]
    if T > 5:
        trees[0][4] = 9                                          # (no earlier node: there is no node 4, nor any that follows it)
    drafted = rng.integers(-1, min(vocab + 1, 40), (n, T)).astype(np.int32)
    history = rng.integers(0, min(vocab, 60), (n, 20)).astype(np.int32)
    length = rng.integers(0, 21, n).astype(np.int32)
    texts = []
    for i in range(n):
        for t in range(T):
            up = M.lineage(trees[i], t) or []
            texts.append(np.concatenate([history[i, :length[i]], drafted[i, up].astype(np.int32)]))
    price = dict(repetition=1.2, presence=0.3, frequency=0.2)
    want, token = apply(logits, texts, **price)
    r = V.token_rules(**price, history=gpu(history), history_len=gpu(length), parents=gpu(np.array(trees, np.int32)), drafted=gpu(drafted))
    check(logits, r, want, token)
    want, token = apply(logits, [x[length[k // T]:] for k, x in enumerate(texts)], **price)
    check(logits, V.token_rules(**price, parents=gpu(np.array(trees, np.int32)), drafted=gpu(drafted)), want, token)


def test_offsets_beyond_32_bits():
    import torch
    vocab, stride = 5000, (1 << 31) // 2 + 8
    wide = torch.empty(2 * stride + vocab, device=DEV)
    x = wide.as_strided((3, vocab), (stride, 1))
    logits = np.random.default_rng(1).standard_normal((3, vocab)).astype(F)
    x.copy_(gpu(logits))
    want, token = apply(logits, [[1, 2]] * 3, frequency=3.0)
    r = V.token_rules(frequency=3.0, history=gpu(np.array([[1, 2]] * 3, np.int32)), history_len=gpu(np.array([2, 2, 2], np.int32)))
    ws = torch.empty(V.vlac_choose_workspace_bytes(3, vocab), dtype=torch.uint8, device=DEV)
    tok = torch.zeros(3, dtype=torch.int32, device=DEV)
    V.vlac_choose_tokens(x, r, x, tok, ws)
    assert same(x.cpu().numpy(), want) and tok.tolist() == token.tolist()


def test_the_binding_checks_sizes():
    import torch
    x = torch.zeros((6, 100), device=DEV)
    ws, tok = torch.empty(4096, dtype=torch.uint8, device=DEV), torch.zeros(6, dtype=torch.int32, device=DEV)
    i = lambda *s: torch.zeros(s, dtype=torch.int32, device=DEV)
    for bad in (lambda: V.token_rules(bias=torch.zeros(99, device=DEV)), lambda: V.token_rules(bias=torch.zeros((5, 100), device=DEV)),
                lambda: V.token_rules(allowed=i(3)), lambda: V.token_rules(allowed=i(5, 4)),
                lambda: V.token_rules(history=i(5, 9), history_len=i(5)), lambda: V.token_rules(parents=i(2, 2), drafted=i(2, 2))):
        with pytest.raises(ValueError):
            V.vlac_choose_tokens(x, bad(), x, tok, ws)
    with pytest.raises(ValueError):
        V.token_rules(history=i(5, 9), history_len=i(6))
    with pytest.raises(ValueError):
        V.token_rules(parents=i(5, 9), drafted=i(5, 8))
    with pytest.raises(TypeError):
        V.token_rules(bias=i(100))
    with pytest.raises(TypeError):
        V.token_rules(allowed=torch.zeros(4, device=DEV))
    with pytest.raises(TypeError):
        V.vlac_choose_tokens(x.half(), V.token_rules(), x, tok, ws)
    with pytest.raises(ValueError):
        V.vlac_choose_tokens(x.t(), V.token_rules(), None, tok, ws)
    with pytest.raises(ValueError):
        V.vlac_choose_tokens(x, V.token_rules(), x, tok[:5], ws)
    with pytest.raises(V.VlacError):
        V.vlac_choose_tokens(x, V.token_rules(), x, tok, ws[:16])


@pytest.mark.parametrize("price", [dict(repetition=1.3), dict(repetition=0.25, presence=1e-40), dict(repetition=3.0, frequency=1e-39)])
def test_the_ends_of_fp32(price):
    """Subnormal logits and penalties, quotients and products that leave the range."""
    rng = np.random.default_rng(6)
    rows, vocab = 3, 3000
    x = np.exp(rng.uniform(-103, 88.7, (rows, vocab))).astype(F) * rng.choice([-1, 1], (rows, vocab)).astype(F)
    x[:, :4] = [3e38, -3e38, 1e-45, -1e-45]
    text = rng.permutation(vocab)[:1500].tolist() + [0, 1, 2, 3]
    want, token = apply(x, [text] * rows, **price)
    r = V.token_rules(**price, history=gpu(np.array([text] * rows, np.int32)), history_len=gpu(np.full(rows, len(text), np.int32)))
    check(x, r, want, token)


def test_the_largest_vocabulary():
    import torch
    vocab = 1 << 24
    x = torch.randn((1, vocab), device=DEV)
    x[0, vocab - 1], x[0, 7] = 99.0, 98.5
    r = V.token_rules(frequency=1.0, history=gpu(np.array([[vocab - 1, 7, vocab, -1]], np.int32)), history_len=gpu(np.array([1], np.int32)))
    ws, tok, out = torch.empty(V.vlac_choose_workspace_bytes(1, vocab), dtype=torch.uint8, device=DEV), torch.zeros(1, dtype=torch.int32, device=DEV), torch.empty_like(x)
    V.vlac_choose_tokens(x, r, out, tok, ws)
    assert tok.item() == 7 and out[0, vocab - 1].item() == 98.0 and bool((out[0, :-1] == x[0, :-1]).all())
    x[0, vocab - 1] = 100.0
    V.vlac_choose_tokens(x, r, None, tok, ws)
    assert tok.item() == vocab - 1


def test_many_rows():
    """More rows than a launch of whole pieces would have threads for in one dimension, two tokens each."""
    import torch
    rows = 1 << 20
    x = torch.randn((rows, 2), device=DEV)
    ws, tok = torch.empty(V.vlac_choose_workspace_bytes(rows, 2), dtype=torch.uint8, device=DEV), torch.zeros(rows, dtype=torch.int32, device=DEV)
    V.vlac_choose_tokens(x, V.token_rules(), None, tok, ws)
    assert torch.equal(tok, (x[:, 1] > x[:, 0]).int())


def test_the_longest_text():
    """2^31 - 1 tokens, 8 GB: the place behind the last turn of the count is beyond 31 bits."""
    import torch
    most, vocab = (1 << 31) - 1, 70
    text = torch.full((1, most), -1, dtype=torch.int32, device=DEV)
    text[0, 0] = text[0, most - 1] = text[0, 1 << 30] = 9
    text[0, most - 300] = 69
    x = torch.zeros((1, vocab), device=DEV)
    x[0, 9] = 3.5
    x[0, 8] = 0.25
    ws, tok = torch.empty(256, dtype=torch.uint8, device=DEV), torch.zeros(1, dtype=torch.int32, device=DEV)
    want = x.clone()
    want[0, 9], want[0, 69] = 3.5 - 3 * 1.25, -1.25
    V.vlac_choose_tokens(x, V.token_rules(frequency=1.25, history=text, history_len=gpu(np.array([most], np.int32))), x, tok, ws)
    assert torch.equal(x, want) and tok.item() == 8


def test_empty_texts_and_batches():
    """History without columns is no text (penalties then hit the drafts alone); a batch without entries is nothing to do."""
    import torch
    i = lambda *s: torch.zeros(s, dtype=torch.int32, device=DEV)
    x = torch.tensor([[1.0, 0.5, 0.25], [1.0, 0.5, 2.0]], device=DEV)
    ws, tok = torch.empty(256, dtype=torch.uint8, device=DEV), i(2)
    out = torch.empty_like(x)
    V.vlac_choose_tokens(x, V.token_rules(presence=9.0, history=i(2, 0), history_len=i(2) + 7), out, tok, ws)
    assert torch.equal(out, x) and tok.tolist() == [0, 2]
    trees = dict(parents=gpu([[-1, 0]], torch.int32), drafted=gpu([[0, 2]], torch.int32))
    V.vlac_choose_tokens(x, V.token_rules(presence=9.0, history=i(1, 0), history_len=i(1), **trees), out, tok, ws)
    assert out.tolist() == [[-8.0, 0.5, 0.25], [-8.0, 0.5, -7.0]] and tok.tolist() == [1, 1]
    with pytest.raises(ValueError):
        V.vlac_choose_tokens(x, V.token_rules(history=i(3, 0), history_len=i(3)), out, tok, ws)
    none = torch.empty((0, 3), device=DEV)
    V.vlac_choose_tokens(none, V.token_rules(presence=1.0, history=i(0, 4), history_len=i(0), parents=i(0, 5), drafted=i(0, 5)), none, i(0), ws)
    with pytest.raises(V.VlacError):
        V.vlac_choose_tokens(x, V.token_rules(parents=i(2, 0), drafted=i(2, 0)), out, tok, ws)
