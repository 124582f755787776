"""Decoding several candidates of one observation over pages: prefill, import, fork, decode, against the oracle (which decodes
every candidate over a cache of its own) with the tolerance of the other decode tests."""
import copy

import numpy as np
import pytest

import synth
import paper_2502_02175_amd as V
from oracle import vlac_oracle as O
from helpers import GpuModel, oracle_model
from pages_model import E_NOMEM, E_RANGE, OK, pages_of

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TOL = 2e-2
GQA = synth.ModelCfg(3, 256, 8, 2, 128, 352, 320, rope_base=1.0e6)


def i32(x):
    import torch
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def margin(x):
    s = np.sort(np.asarray(x, dtype=np.float64))
    return s[-1] - s[-2]


def decode(gm, pool, seqs, L, n_new, first, group):
    import torch
    n = len(seqs)
    ws = torch.empty(V.vlac_candidates_workspace_bytes(gm.ctx, pool, n), dtype=torch.uint8, device=DEV)
    toks = torch.full((n, n_new), -7, dtype=torch.int32, device=DEV)
    logits = torch.full((n, n_new, gm.cfg.vocab), float("nan"), device=DEV)
    V.vlac_decode_candidates(gm.ctx, pool, i32(seqs), n, L, None if group is None else i32(group), n_new, i32(first), toks,
                             logits, ws)
    return toks.cpu().numpy(), logits.cpu().numpy()


@pytest.mark.parametrize("cfg,operand,B,each,L", [
    (synth.CONFIGS["tiny"], "f16", 1, 4, 64),       # norms fused into the projections; a page boundary at once
    (synth.CONFIGS["tiny"], "f16", 2, 8, 59),       # 16 rows, the boundary after five tokens
    (GQA, "f16", 2, 3, 33),
    (GQA, "f16", 3, 14, 70),                        # 42 rows: the prefill's projections
    (synth.CONFIGS["tiny"], "f16w8", 2, 2, 31),
    (synth.CONFIGS["tiny"], "bf16", 1, 6, 40),
])
def test_candidates_against_the_oracle(cfg, operand, B, each, L):
    n_new, n = 7, B * each
    om = oracle_model(cfg, seed=3, std=0.05, w8=operand == "f16w8")
    gm = GpuModel(cfg, seed=3, max_batch=max(n, B), max_seq=96, std=0.05, operand=operand)
    try:
        rng = np.random.default_rng(8)
        emb = synth.round_bf16(rng.standard_normal((B, L, cfg.d_model)))
        gm.prefill(emb, L - 11)
        caches = []
        for b in range(B):
            caches.append(O.new_cache(cfg, 96))
            O.dense_forward(om, emb[b], L - 11, caches[b])
        pool = V.new_pages(cfg.n_layers, cfg.n_kv_heads, cfg.head_dim, gm.ccfg.operand_dtype,
                           B * pages_of(L) + n * (1 + pages_of(L % 32 + n_new)) + 2, B + n, 3, DEV)
        pool.tensors[0].fill_(0xFF)                           # NaN where nothing was written
        V.vlac_pages_import(gm.ctx, gm.kv, B, L, pool, i32(range(B)))
        src = [b for b in range(B) for _ in range(each)]
        seqs = list(range(B, B + n))
        first = rng.integers(0, cfg.vocab, n).tolist()        # what a sampler would draw
        V.vlac_pages_fork(pool, i32(src), i32(seqs), n)
        keep = gm.kv.clone()
        gt, gl = decode(gm, pool, seqs, L, n_new, first, src)
        assert V.vlac_pages_check(pool, check=False) == OK
        assert bool((gm.kv == keep).all())                    # the streams' cache is not touched
        assert pool.tensors[3].tolist() == [L] * B + [L + n_new] * n
        worst = compared = 0
        for i in range(n):
            toks, logits = O.decode(om, copy.deepcopy(caches[src[i]]), L, first[i], n_new, return_logits=True)
            ok = 0
            for t in range(n_new):                             # (a greedy choice within the tolerance may part the two)
                worst = max(worst, np.abs(gl[i, t] - logits[t]).max())
                if margin(logits[t]) <= 2 * TOL:
                    break
                assert int(gt[i, t]) == toks[t], (i, t)
                compared += 1
        assert worst <= TOL, worst
        assert compared >= n * n_new // 3
        # once more over the same sources: the same bits, and again with no groups within the tolerance of rounding
        V.vlac_pages_fork(pool, i32(src), i32(seqs), n)
        gt2, gl2 = decode(gm, pool, seqs, L, n_new, first, src)
        assert (gt2 == gt).all() and np.array_equal(gl2, gl)
        V.vlac_pages_free(pool, i32(range(B + n)), B + n)
        assert not bool(pool.tensors[1].any()) and V.vlac_pages_check(pool, check=False) == OK
    finally:
        gm.close()


def test_a_candidate_decodes_what_the_stream_decodes():
    """The greedy first token: both ways to decode are within TOL of the oracle, so within 2 TOL of each other."""
    cfg, L, n_new = synth.CONFIGS["tiny"], 75, 6
    gm = GpuModel(cfg, seed=5, max_batch=3, max_seq=96, std=0.05)
    try:
        emb = synth.round_bf16(np.random.default_rng(1).standard_normal((2, L, cfg.d_model)))
        got = gm.prefill(emb, 64)
        pool = V.new_pages(cfg.n_layers, cfg.n_kv_heads, cfg.head_dim, 1, 20, 5, 3, DEV)
        V.vlac_pages_import(gm.ctx, gm.kv, 2, L, pool, i32([0, 1]))
        st, sl = gm.decode(2, L, n_new, got["token"])
        V.vlac_pages_fork(pool, i32([1, 0]), i32([2, 3]), 2)
        ct, cl = decode(gm, pool, [2, 3], L, n_new, got["token"][::-1].tolist(), [1, 0])
        same = [b for b in range(2) if (ct[1 - b] == st[b]).all()]
        assert same
        for b in same:
            assert np.abs(cl[1 - b] - sl[b]).max() <= 2 * TOL
    finally:
        gm.close()


def test_refusals_and_reports():
    import torch
    cfg, L = synth.CONFIGS["tiny"], 40
    gm = GpuModel(cfg, seed=5, max_batch=4, max_seq=64, std=0.05)
    try:
        emb = synth.round_bf16(np.random.default_rng(1).standard_normal((1, L, cfg.d_model)))
        gm.prefill(emb, 32)
        make = lambda n_pages=20, op=1, layers=cfg.n_layers, heads=cfg.n_kv_heads, cols=3: V.new_pages(
            layers, heads, cfg.head_dim, op, n_pages, 6, cols, DEV)
        pool = make()
        V.vlac_pages_import(gm.ctx, gm.kv, 1, L, pool, i32([0]))
        ws = torch.empty(V.vlac_candidates_workspace_bytes(gm.ctx, pool, 4), dtype=torch.uint8, device=DEV)
        toks = torch.full((4, 8), -7, dtype=torch.int32, device=DEV)
        four = i32([1, 2, 3, 4])

        def call(p=pool, seqs=four, n=4, L=L, n_new=3, first=four, out=toks, w=ws):
            return V.vlac_decode_candidates(gm.ctx, p, seqs, n, L, None, n_new, first, out, None, w, check=False)

        V.vlac_pages_fork(pool, i32([0] * 4), four, 4)
        before = [x.clone() for x in pool.tensors]
        assert call(n=-1) == E_RANGE and call(seqs=i32([0] * 5), first=i32([0] * 5), n=5, n_new=1) == E_RANGE
        assert call(L=0) == E_RANGE and call(n_new=-1) == E_RANGE
        assert call(L=60, n_new=5) == -2                           # max_seq 64
        assert call(p=make(op=0)) == -2 and call(p=make(layers=1)) == -2 and call(p=make(heads=2)) == -2
        assert call(p=make(cols=1)) == -2                          # 43 positions on one page
        assert call(seqs=None) == -1 and call(first=None) == -1 and call(out=None) == -1 and call(w=None) == -1
        assert call(w=ws[:100]) == E_RANGE and call(w=ws[4:]) == -2
        assert call(n=0) == OK and call(n_new=0) == OK
        assert V.vlac_candidates_workspace_bytes(gm.ctx, pool, 5) == 0 and V.vlac_candidates_workspace_bytes(gm.ctx, make(op=0), 4) == 0
        torch.cuda.synchronize()
        assert all(bool((x == y).all()) for x, y in zip(pool.tensors, before)) and bool((toks == -7).all())
        # a sequence of another length, one that does not exist, one listed twice: the others decode
        V.vlac_pages_extend(pool, i32([2]), 1, 1, i32([0]))
        assert call(seqs=i32([1, 2, 99, 1])) == OK
        assert V.vlac_pages_check(pool, check=False) == E_RANGE
        assert pool.tensors[3].tolist() == [40, 43, 41, 40, 40, 0]
        want = toks[0, :3].clone()
        V.vlac_pages_fork(pool, i32([0] * 4), four, 4)
        assert call() == OK and bool((toks.view(-1)[:3] == want).all())
        # no room: the sequences stay
        tight = make(n_pages=6)                                    # 2 + 4 last pages, none for the 65th position
        V.vlac_pages_import(gm.ctx, gm.kv, 1, L, tight, i32([0]))
        V.vlac_pages_fork(tight, i32([0] * 4), four, 4)
        assert V.vlac_pages_check(tight, check=False) == OK
        more = torch.full((4, 24), -7, dtype=torch.int32, device=DEV)
        assert call(p=tight, n_new=24, out=more) == OK and V.vlac_pages_check(tight, check=False) == OK     # 64 positions: no new page
        V.vlac_pages_fork(tight, i32([0] * 4), four, 4)
        V.vlac_pages_extend(tight, four, 4, 25, i32([0] * 4))
        assert V.vlac_pages_check(tight, check=False) == E_NOMEM and tight.tensors[3].tolist() == [40, 40, 40, 40, 40, 0]
    finally:
        gm.close()


def test_decoding_captured_in_a_graph():
    """Fork and decode in one graph, replayed between eager decodes of the streams on the same context."""
    import torch
    cfg, L, n_new, n = synth.CONFIGS["tiny"], 60, 5, 6
    gm = GpuModel(cfg, seed=5, max_batch=n, max_seq=96, std=0.05)
    try:
        rng = np.random.default_rng(1)
        got = gm.prefill(synth.round_bf16(rng.standard_normal((2, L, cfg.d_model))), 48)
        pool = V.new_pages(cfg.n_layers, cfg.n_kv_heads, cfg.head_dim, 1, 24, 2 + n, 3, DEV)
        V.vlac_pages_import(gm.ctx, gm.kv, 2, L, pool, i32([0, 1]))
        src, seqs, first = i32([0, 0, 0, 1, 1, 1]), i32(range(2, 2 + n)), i32([3, 9, 27, 81, 243, 11])
        toks = torch.zeros((n, n_new), dtype=torch.int32, device=DEV)
        logits = torch.zeros((n, n_new, cfg.vocab), device=DEV)
        ws = torch.empty(V.vlac_candidates_workspace_bytes(gm.ctx, pool, n), dtype=torch.uint8, device=DEV)

        def work():
            V.vlac_pages_fork(pool, src, seqs, n)
            V.vlac_decode_candidates(gm.ctx, pool, seqs, n, L, src, n_new, first, toks, logits, ws)

        work()
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            work()
        for r in range(3):
            first.copy_(torch.randint(0, cfg.vocab, (n,), device=DEV).int())
            work()
            torch.cuda.synchronize()
            want = toks.clone(), logits.clone()
            toks.fill_(-7)
            logits.zero_()
            gm.decode(2, L, n_new, got["token"])                # (the context's buffers hold other rows)
            g.replay()
            torch.cuda.synchronize()
            assert bool((toks == want[0]).all()) and bool((logits == want[1]).all()), r
        assert V.vlac_pages_check(pool, check=False) == OK
    finally:
        gm.close()
