"""Decoding candidates without groups against the oracle, and in a pool that has no page left for them."""
import copy

import numpy as np
import pytest

import synth
import paper_2502_02175_amd as V
from oracle import vlac_oracle as O
from helpers import GpuModel, oracle_model
from pages_model import E_NOMEM, OK, pages_of
from test_gpu_candidates import DEV, GQA, TOL, decode, i32, margin

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("cfg,operand,each,L,group", [
    (synth.CONFIGS["tiny"], "f16", 2, 62, None),                        # (two observations in what is taken for one group)
    (synth.CONFIGS["tiny"], "bf16", 5, 40, None),
    (GQA, "f16", 4, 35, None),
    (GQA, "f16", 18, 64, None),
    (GQA, "f16", 3, 35, [7, 1, 7, 1, 7, 1]),                            # candidates of the observations in turn
])
def test_groups_make_no_difference_to_the_oracle(cfg, operand, each, L, group):
    B, n_new = 2, 5
    n = B * each
    om = oracle_model(cfg, seed=3, std=0.05)
    gm = GpuModel(cfg, seed=3, max_batch=n, max_seq=96, std=0.05, operand=operand)
    try:
        rng = np.random.default_rng(9)
        emb = synth.round_bf16(rng.standard_normal((B, L, cfg.d_model)))
        gm.prefill(emb, L - 11)
        caches = []
        for b in range(B):
            caches.append(O.new_cache(cfg, 96))
            O.dense_forward(om, emb[b], L - 11, caches[b])
        pool = V.new_pages(cfg.n_layers, cfg.n_kv_heads, cfg.head_dim, gm.ccfg.operand_dtype,
                           B * pages_of(L) + n * (1 + pages_of(L % 32 + n_new)) + 2, B + n, 3, DEV)
        pool.tensors[0].fill_(0xFF)
        V.vlac_pages_import(gm.ctx, gm.kv, B, L, pool, i32(range(B)))
        src = [i % B for i in range(n)]
        seqs, first = list(range(B, B + n)), rng.integers(0, cfg.vocab, n).tolist()
        V.vlac_pages_fork(pool, i32(src), i32(seqs), n)
        gt, gl = decode(gm, pool, seqs, L, n_new, first, group)
        assert V.vlac_pages_check(pool, check=False) == OK
        compared = 0
        for i in range(n):
            toks, logits = O.decode(om, copy.deepcopy(caches[src[i]]), L, first[i], n_new, return_logits=True)
            for t in range(n_new):
                assert np.abs(gl[i, t] - logits[t]).max() <= TOL, (i, t)
                if margin(logits[t]) <= 2 * TOL:                # (a greedy choice within the tolerance may part the two)
                    break
                assert int(gt[i, t]) == toks[t], (i, t)
                compared += 1
        assert compared >= n * n_new // 3
    finally:
        gm.close()


@pytest.mark.parametrize("n", [2, 4, 6])
def test_no_room_for_the_new_tokens(n):
    """The prefill ends at a page's end and the pool is full: nothing is decoded, and nothing but the outputs is touched."""
    import torch
    cfg, L = synth.CONFIGS["tiny"], 64
    gm = GpuModel(cfg, seed=5, max_batch=n, max_seq=96, std=0.05)
    try:
        emb = synth.round_bf16(np.random.default_rng(1).standard_normal((1, L, cfg.d_model)))
        gm.prefill(emb, 48)
        pool = V.new_pages(cfg.n_layers, cfg.n_kv_heads, cfg.head_dim, 1, 2 + n - 1, 1 + n, 3, DEV)
        pool.tensors[0].fill_(0xFF)
        V.vlac_pages_import(gm.ctx, gm.kv, 1, L, pool, i32([0]))
        seqs = list(range(1, 1 + n))
        V.vlac_pages_fork(pool, i32([0] * n), i32(seqs), n)     # (no copies: every page is full)
        assert V.vlac_pages_check(pool, check=False) == OK
        before = [x.clone() for x in pool.tensors[:4]]
        keep = gm.kv.clone()
        decode(gm, pool, seqs, L, 7, [3] * n, None)
        assert V.vlac_pages_check(pool, check=False) == E_NOMEM and V.vlac_pages_check(pool, check=False) == OK
        assert all(bool((x == y).all()) for x, y in zip(pool.tensors, before)) and bool((gm.kv == keep).all())
        # one candidate less has room, and the pool decodes as ever
        toks, logits = decode(gm, pool, seqs[:-1], L, 7, [3] * (n - 1), None)
        assert V.vlac_pages_check(pool, check=False) == OK and np.isfinite(logits).all()
        assert (toks == toks[0]).all() and pool.tensors[3].tolist() == [L] + [L + 7] * (n - 1) + [L]
        torch.cuda.synchronize()
    finally:
        gm.close()
