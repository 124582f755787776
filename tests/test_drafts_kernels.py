"""How many kernels on drafted tokens the built library has of every name: what their registers are held against has to find them all."""
import pytest

from test_pages_registers import of

COUNTS = {
    "rotary_append_kernel": 2 * 2 * 4 * 3,   # head sizes, types, ways to turn, heads of a wave
    "rotary_fill_kernel": 1,
    "attend_tree_kernel": 4, "attend_tree_few_kernel": 4, "attend_tree_join_kernel": 4,   # head sizes, types
    "attend_tree_mask_kernel": 1,
    "choose_kernel": 2 * 2,                  # with and without texts, logits of a thread
    "choose_join_kernel": 1, "tree_accept_kernel": 1, "pages_keep_kernel": 1, "pages_keep_end_kernel": 1}


@pytest.mark.parametrize("name", sorted(COUNTS))
def test_every_kernel_is_found(name):
    mine = of(name)
    assert len(mine) == COUNTS[name]
    for n, k in mine.items():
        assert k[".private_segment_fixed_size"] == 0 and k[".vgpr_spill_count"] == 0, n
