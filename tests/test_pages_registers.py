"""Registers of the kernels on pages, from the metadata of the built library: the attention holds a column block's queries, keys,
values and sums in registers and has 256 of them per lane (two waves per SIMD); one more would be a spill in its
loop, which no result shows."""
from test_registers import kernels


def of(*names):
    return {n: k for n, k in kernels().items() if any("%d%s" % (len(x), x) in n for x in names)}


def test_the_attention_over_pages_does_not_spill():
    mine = of("attend_kernel")
    assert len(mine) == 4                                    # head sizes, types
    for n, k in mine.items():
        assert k[".private_segment_fixed_size"] == 0 and k[".vgpr_spill_count"] == 0 and k[".vgpr_count"] <= 256, n
        assert k[".group_segment_fixed_size"] <= 160 * 1024, n


def test_nor_does_the_one_for_few_columns():
    mine = of("attend_few_kernel")
    assert len(mine) == 4
    for n, k in mine.items():
        assert k[".private_segment_fixed_size"] == 0 and k[".vgpr_spill_count"] == 0 and k[".vgpr_count"] <= 256, n


def test_nor_does_any_other_kernel_on_pages():
    mine = of("attend_plan_kernel", "attend_join_kernel", "pages_plan_kernel", "pages_copy_kernel", "pages_import_kernel",
              "pages_reset_kernel", "pages_free_kernel", "pages_compact_kernel", "pages_append_kernel")
    assert len(mine) == 2 + 4 + 3 + 2 + 1 + 1 + 1 + 1 + 2
    for n, k in mine.items():
        assert k[".private_segment_fixed_size"] == 0 and k[".vgpr_spill_count"] == 0, n
        assert k[".group_segment_fixed_size"] <= 160 * 1024, n
