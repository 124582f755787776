"""More new rows in one call than a launch may have threads for."""
import pytest

import paper_2502_02175_amd as V
from pages_model import E_RANGE, PAGE, k_tile_at, v_tile_at
from test_gpu_pages import i32

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def test_append_of_a_very_long_chunk():
    """2^18 tokens of 1024 kv heads of 128 (64 GiB): 2^32 threads and more.  Only the last page of the sequence is there; the
    places before it name none, and are reported."""
    import torch
    T, heads, hd = 1 << 18, 1024, 128
    if torch.cuda.mem_get_info()[0] < 80 << 30:
        pytest.skip("64 GiB of rows do not fit beside what is held")
    p = V.new_pages(1, heads, hd, 1, 3, 1, T // PAGE, DEV)
    data, refs, table, length, _ = p.tensors
    data.fill_(0x5A)
    table[0, -1] = 1
    refs[1] = 1
    length[0] = T
    rows = torch.empty((1, T, heads, hd), dtype=torch.float16, device=DEV)
    last = rows[0, -PAGE:]
    last.copy_(torch.randn(last.shape, device=DEV))
    try:
        assert V.vlac_pages_append(p, 0, i32([0]), i32([0]), 1, T, rows, rows, check=False) == 0
        assert V.vlac_pages_check(p, check=False) == E_RANGE
        d = data.view(torch.int16).view(3, 2, heads, PAGE * hd)
        assert bool((d[0] == 0x5A5A).all()) and bool((d[2] == 0x5A5A).all())
        x = last.view(torch.int16).permute(1, 0, 2).reshape(heads, PAGE * hd)
        for which, at in ((0, k_tile_at(hd)), (1, v_tile_at(hd))):
            assert bool((d[1, which][:, torch.tensor(at, device=DEV).flatten()] == x).all()), which
    finally:
        del rows, last
        torch.cuda.empty_cache()
