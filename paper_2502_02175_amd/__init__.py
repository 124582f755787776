"""vlac: VLA-Cache sparse prefill on MI355X.  Thin ctypes binding over the C ABI
declared in include/vlac.h; every computation runs in libvlac.so's HIP kernels."""
from .binding import (VlacError, ModelCfg, LayerW, OPERAND_BF16, OPERAND_F16, OPERAND_F16_W8, lib, lib_path, use_library, status_string,
                      vlac_create, vlac_destroy, vlac_set_layer_weights, vlac_set_head_weights,
                      vlac_kv_cache_bytes, vlac_plan_many_rows_gemm, vlac_plan_unsplit_gemm, vlac_reset_stream, vlac_check, vlac_select_static, vlac_select_static_noalloc, vlac_embed_patches, vlac_quantize_e4m3,
                      vlac_layer_ratio, vlac_sparse_prefill, vlac_decode_action,
                      vlac_last_hip_error, vlac_profile_select, vlac_profile_read,
                      vlac_profile_read2, vlac_profile_bracket_cost,
                      Pages, pages, new_pages, vlac_page_bytes, vlac_pages_scratch_bytes, vlac_pages_reset, vlac_pages_check,
                      vlac_pages_import, vlac_pages_fork, vlac_pages_extend, vlac_pages_append, vlac_pages_free,
                      vlac_pages_compact, vlac_attend_workspace_bytes, vlac_attend_plan, vlac_attend_shared, vlac_plan_attention,
                      vlac_candidates_workspace_bytes, vlac_decode_candidates,
                      Rotary, rotary, ROTARY_HALF, ROTARY_PAIRS, vlac_rotary_fill, vlac_pages_append_rotated, TREE_MAX_NODES,
                      vlac_attend_tree_workspace_bytes, vlac_attend_tree_plan, vlac_attend_tree, TokenRules, token_rules,
                      vlac_choose_workspace_bytes, vlac_choose_tokens, vlac_tree_accept, vlac_pages_keep,
                      vlac_guided_workspace_bytes, vlac_decode_guided)

__all__ = [n for n in dir() if n.startswith("vlac_")] + [
    "VlacError", "ModelCfg", "LayerW", "OPERAND_BF16", "OPERAND_F16", "OPERAND_F16_W8", "lib", "lib_path", "use_library", "status_string", "Pages", "pages", "new_pages",
    "Rotary", "rotary", "ROTARY_HALF", "ROTARY_PAIRS", "TREE_MAX_NODES", "TokenRules", "token_rules"]
