"""Tensors that are too small for what a call reads or writes are refused by the binding, before anything is queued."""
import pytest

import synth
import paper_2502_02175_amd as V
from helpers import GpuModel
from test_gpu_candidates import i32

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def test_a_cache_or_logits_of_too_few_values():
    import torch
    cfg = synth.CONFIGS["tiny"]
    gm = GpuModel(cfg, seed=5, max_batch=4, max_seq=64, std=0.05)
    try:
        pool = V.new_pages(cfg.n_layers, cfg.n_kv_heads, cfg.head_dim, 1, 20, 6, 3, DEV)
        before = [x.clone() for x in pool.tensors]
        size = gm.kv.numel()
        assert size == V.vlac_kv_cache_bytes(gm.ccfg)
        with pytest.raises(ValueError):
            V.vlac_pages_import(gm.ctx, gm.kv[:size - 16], 1, 40, pool, i32([0]), check=False)
        # (whole in bytes of another type; and no prefill was made: the status of the call itself)
        assert V.vlac_pages_import(gm.ctx, gm.kv.view(torch.float16), 1, 40, pool, i32([0]), check=False) == -4
        n, n_new = 3, 2
        ws = torch.empty(V.vlac_candidates_workspace_bytes(gm.ctx, pool, n), dtype=torch.uint8, device=DEV)
        toks = torch.full((n, n_new), -7, dtype=torch.int32, device=DEV)

        def call(logits):
            return V.vlac_decode_candidates(gm.ctx, pool, i32([1, 2, 3]), n, 40, None, n_new, i32([0] * 3), toks, logits, ws,
                                            check=False)

        with pytest.raises(ValueError):
            call(torch.zeros(n * n_new * cfg.vocab - 1, device=DEV))
        with pytest.raises(ValueError):
            call(torch.zeros((n, cfg.vocab), device=DEV))
        with pytest.raises(TypeError):
            call(torch.zeros((n, n_new, cfg.vocab), dtype=torch.float16, device=DEV))
        torch.cuda.synchronize()
        assert all(bool((x == y).all()) for x, y in zip(pool.tensors, before)) and bool((toks == -7).all())
        assert call(torch.zeros((n, n_new, cfg.vocab), device=DEV)) == 0
        assert V.vlac_pages_check(pool, check=False) == -3      # (no sequence has 40 positions)
    finally:
        gm.close()
