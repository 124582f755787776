"""Decoding candidates under rules: with rules that change nothing the bits of vlac_decode_candidates, with others the rules' own
arithmetic on the oracle's logits, each candidate fed the tokens that it chose."""
import copy
import math

import numpy as np
import pytest

import synth
import paper_2502_02175_amd as V
from helpers import GpuModel, oracle_model
from oracle import vlac_oracle as O
from pages_model import E_RANGE, OK, pages_of
from test_gpu_candidates import GQA, TOL, decode, i32
from test_gpu_choose import apply, bits, gpu

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def guided(gm, pool, seqs, L, n_new, first, group, rules, logits=True):
    import torch
    n = len(seqs)
    ws = torch.empty(V.vlac_guided_workspace_bytes(gm.ctx, pool, n), dtype=torch.uint8, device=DEV)
    ws.fill_(0xFF)
    toks = torch.full((n, n_new), -7, dtype=torch.int32, device=DEV)
    lg = torch.full((n, n_new, gm.cfg.vocab), float("nan"), device=DEV) if logits else None
    V.vlac_decode_guided(gm.ctx, pool, i32(seqs), n, L, None if group is None else i32(group), n_new, i32(first), rules, toks, lg, ws)
    return toks.cpu().numpy(), lg.cpu().numpy() if logits else None


@pytest.mark.parametrize("cfg,operand,B,each,L", [
    (synth.CONFIGS["tiny"], "f16", 1, 4, 64),       # norms fused into the projections
    (synth.CONFIGS["tiny"], "bf16", 2, 8, 59),
    (GQA, "f16", 3, 14, 70),                        # 42 rows: the prefill's projections
])
def test_against_the_oracle(cfg, operand, B, each, L):
    n_new, n = 6, B * each
    om = oracle_model(cfg, seed=3, std=0.05)
    gm = GpuModel(cfg, seed=3, max_batch=max(n, B), max_seq=96, std=0.05, operand=operand)
    try:
        rng = np.random.default_rng(8)
        emb = synth.round_bf16(rng.standard_normal((B, L, cfg.d_model)))
        gm.prefill(emb, L - 11)
        pool = V.new_pages(cfg.n_layers, cfg.n_kv_heads, cfg.head_dim, gm.ccfg.operand_dtype,
                           B * pages_of(L) + n * (1 + pages_of(L % 32 + n_new)) + 2, B + n, 3, DEV)
        V.vlac_pages_import(gm.ctx, gm.kv, B, L, pool, i32(range(B)))
        src, seqs = [b for b in range(B) for _ in range(each)], list(range(B, B + n))
        first = rng.integers(0, cfg.vocab, n).tolist()

        def fork():
            V.vlac_pages_fork(pool, i32(src), i32(seqs), n)

        fork()
        plain, plain_logits = decode(gm, pool, seqs, L, n_new, first, src)
        fork()
        toks, logits = guided(gm, pool, seqs, L, n_new, first, src, V.token_rules())
        assert np.array_equal(toks, plain) and np.array_equal(logits, plain_logits)
        # rules of every kind: a step's mask differs from the next one's
        price = dict(repetition=1.25, presence=0.2, frequency=0.1)
        history = rng.integers(0, cfg.vocab, (n, 9)).astype(np.int32)
        length = (np.arange(n) % 10).astype(np.int32)
        bias = np.where(rng.random(cfg.vocab) < 0.1, 0.5, 0).astype(np.float32)
        allowed = rng.random((n * n_new, cfg.vocab)) < 0.5
        rules = V.token_rules(**price, bias=gpu(bias), allowed=gpu(bits(allowed)), history=gpu(history), history_len=gpu(length))
        fork()
        toks, logits = guided(gm, pool, seqs, L, n_new, first, src, rules)
        assert V.vlac_pages_check(pool, check=False) == OK
        fork()
        alone, _ = guided(gm, pool, seqs, L, n_new, first, src, rules, logits=False)
        assert np.array_equal(alone, toks)
        caches = []
        for b in range(B):
            caches.append(O.new_cache(cfg, 96))
            O.dense_forward(om, emb[b], L - 11, caches[b])
        for i in range(0, n, 1 if n < 20 else 5):
            text, cache, fed = history[i, :length[i]].tolist(), copy.deepcopy(caches[src[i]]), first[i]
            for t in range(n_new):
                text.append(fed)
                _, raw = O.decode(om, cache, L + t, fed, 1, return_logits=True)
                want, _ = apply(raw[0][None].astype(np.float32), [text], **price, bias=bias[None], allowed=allowed[i * n_new + t][None])
                got = logits[i, t]
                assert np.array_equal(np.isinf(got), ~allowed[i * n_new + t])
                ok = allowed[i * n_new + t]
                # TOL on the raw logits; a penalty multiplies it, and where it meets a sign that rounding decides
                # the two branches are off by |l| (repetition - 1 / repetition) more, |l| <= TOL there
                assert np.abs(got[ok] - want[0][ok]).max() <= TOL * (price["repetition"] * 2)
                fed = int(toks[i, t])
                assert fed == int(np.where(ok, got, -np.inf).argmax())
    finally:
        gm.close()


def test_only_the_bins_of_an_action():
    """A mask for all rows that leaves the last 16 tokens, and no token twice."""
    cfg, L, n_new = synth.CONFIGS["tiny"], 40, 7
    gm = GpuModel(cfg, seed=5, max_batch=4, max_seq=64, std=0.05)
    try:
        gm.prefill(synth.round_bf16(np.random.default_rng(1).standard_normal((1, L, cfg.d_model))), 32)
        pool = V.new_pages(cfg.n_layers, cfg.n_kv_heads, cfg.head_dim, 1, 20, 5, 3, DEV)
        V.vlac_pages_import(gm.ctx, gm.kv, 1, L, pool, i32([0]))
        V.vlac_pages_fork(pool, i32([0, 0, 0]), i32([1, 2, 3]), 3)
        allowed = np.zeros(cfg.vocab, bool)
        allowed[-16:] = True
        first = [3, cfg.vocab - 1, cfg.vocab - 5]
        toks, logits = guided(gm, pool, [1, 2, 3], L, n_new, first, None, V.token_rules(frequency=1e4, allowed=gpu(bits(allowed))))
        for i in range(3):
            assert len({first[i], *toks[i].tolist()}) == n_new + 1 and (toks[i] >= cfg.vocab - 16).all()
            assert np.isinf(logits[i][:, :-16]).all()
        # nothing is allowed in the second step: -1, and decoding goes on
        mask = np.ones((3 * n_new, cfg.vocab), bool)
        mask[1::n_new] = False
        V.vlac_pages_fork(pool, i32([0, 0, 0]), i32([1, 2, 3]), 3)
        toks, logits = guided(gm, pool, [1, 2, 3], L, n_new, first, None, V.token_rules(allowed=gpu(bits(mask))))
        assert (toks[:, 1] == -1).all() and (np.delete(toks, 1, 1) >= 0).all() and np.isfinite(logits[:, 2:]).all()
        V.vlac_pages_fork(pool, i32([0, 0, 0]), i32([1, 2, 3]), 3)
        V.vlac_pages_extend(pool, i32([1, 2, 3]), 3, 1, i32([0, 0, 0]))
        assert V.vlac_pages_check(pool, check=False) == OK
    finally:
        gm.close()


def test_captured_and_replayed():
    """A graph of fork, guided decoding and release, replayed with other masks and first tokens in its buffers."""
    import torch
    cfg, L, n_new, n = synth.CONFIGS["tiny"], 40, 5, 3
    gm = GpuModel(cfg, seed=5, max_batch=4, max_seq=64, std=0.05)
    try:
        gm.prefill(synth.round_bf16(np.random.default_rng(1).standard_normal((1, L, cfg.d_model))), 32)
        pool = V.new_pages(cfg.n_layers, cfg.n_kv_heads, cfg.head_dim, 1, 20, 5, 3, DEV)
        V.vlac_pages_import(gm.ctx, gm.kv, 1, L, pool, i32([0]))
        rng = np.random.default_rng(4)
        src, seqs, first = i32([0] * n), i32([1, 2, 3]), i32([0] * n)
        allowed = torch.full((n * n_new, cfg.vocab // 32), -1, dtype=torch.int32, device=DEV)
        history, length = i32(rng.integers(0, cfg.vocab, (n, 8)).tolist()), i32([8, 3, 0])
        rules = V.token_rules(repetition=1.3, frequency=0.2, allowed=allowed, history=history, history_len=length)
        ws = torch.empty(V.vlac_guided_workspace_bytes(gm.ctx, pool, n), dtype=torch.uint8, device=DEV)
        toks, logits = torch.zeros((n, n_new), dtype=torch.int32, device=DEV), torch.zeros((n, n_new, cfg.vocab), device=DEV)

        def turn():
            V.vlac_pages_fork(pool, src, seqs, n)
            V.vlac_decode_guided(gm.ctx, pool, seqs, n, L, None, n_new, first, rules, toks, logits, ws)
            V.vlac_pages_free(pool, seqs, n)

        turn()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            turn()
        for k in range(4):
            allowed.copy_(gpu(bits(rng.random((n * n_new, cfg.vocab)) < 0.4)))
            first.copy_(i32(rng.integers(0, cfg.vocab, n).tolist()))
            graph.replay()
            got = toks.clone(), logits.clone()
            turn()
            assert torch.equal(got[0], toks) and torch.equal(got[1], logits)
            assert V.vlac_pages_check(pool, check=False) == OK
    finally:
        gm.close()


def test_refusals():
    import torch
    cfg, L = synth.CONFIGS["tiny"], 40
    gm = GpuModel(cfg, seed=5, max_batch=4, max_seq=64, std=0.05)
    try:
        gm.prefill(synth.round_bf16(np.random.default_rng(1).standard_normal((1, L, cfg.d_model))), 32)
        pool = V.new_pages(cfg.n_layers, cfg.n_kv_heads, cfg.head_dim, 1, 20, 5, 3, DEV)
        V.vlac_pages_import(gm.ctx, gm.kv, 1, L, pool, i32([0]))
        toks = torch.zeros((1, 30), dtype=torch.int32, device=DEV)
        size = V.vlac_guided_workspace_bytes(gm.ctx, pool, 1)
        ws = torch.empty(size, dtype=torch.uint8, device=DEV)
        assert size > V.vlac_candidates_workspace_bytes(gm.ctx, pool, 1)

        def status(rules, ws=ws, n=1, L=L, n_new=3):
            return V.vlac_decode_guided(gm.ctx, pool, i32([0]), n, L, None, n_new, i32([0]), rules, toks, None, ws, check=False)

        assert status(None) == -1
        assert status(V.token_rules(repetition=0.0)) == E_RANGE and status(V.token_rules(presence=math.nan)) == E_RANGE
        tree = i32([[-1, 0]])
        with pytest.raises(V.VlacError):
            V.vlac_decode_guided(gm.ctx, pool, i32([0]), 1, L, None, 3, i32([0]), V.token_rules(parents=tree, drafted=tree), toks, None, ws)
        assert status(V.token_rules(), ws=ws[:size - 256]) == E_RANGE
        assert status(V.token_rules(), n_new=30) == -2 and status(V.token_rules(), L=0) == E_RANGE
        with pytest.raises(ValueError):
            status(V.token_rules(bias=torch.zeros(cfg.vocab + 1, device=DEV)))
        with pytest.raises(ValueError):
            status(V.token_rules(allowed=torch.zeros((2, cfg.vocab // 32), dtype=torch.int32, device=DEV)))
        assert V.vlac_pages_check(pool, check=False) == OK and pool.tensors[3].tolist()[0] == L
        assert status(V.token_rules(), n=0) == 0 and status(V.token_rules(), n_new=0) == 0
    finally:
        gm.close()
