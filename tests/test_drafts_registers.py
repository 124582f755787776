"""Registers and LDS of the kernels on drafted tokens, from the metadata of the built library."""
from test_pages_registers import of


def test_the_attention_of_trees_does_not_spill():
    mine = of("attend_tree_kernel", "attend_tree_few_kernel")
    assert len(mine) == 8                                    # head sizes, types
    for n, k in mine.items():
        assert k[".private_segment_fixed_size"] == 0 and k[".vgpr_spill_count"] == 0 and k[".vgpr_count"] <= 256, n
        assert k[".group_segment_fixed_size"] <= 160 * 1024, n


def test_nor_does_any_other_kernel_on_drafts():
    mine = of("attend_tree_join_kernel", "attend_tree_mask_kernel", "rotary_append_kernel", "rotary_fill_kernel", "choose_kernel",
              "choose_join_kernel", "tree_accept_kernel", "pages_keep_kernel", "pages_keep_end_kernel")
    assert len(mine) >= 4 + 1 + 4 + 1 + 2 + 1 + 1 + 1 + 1
    for n, k in mine.items():
        assert k[".private_segment_fixed_size"] == 0 and k[".vgpr_spill_count"] == 0, n
        assert k[".group_segment_fixed_size"] <= 64 * 1024, n
