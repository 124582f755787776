"""The binding over a pool of bare addresses (a vlac_pages that the caller filled in), without a GPU: every call reaches the library,
whose refusals come back, and host tensors are refused."""
import pytest

import paper_2502_02175_amd as V
from test_pages_abi import FAKE, pool

E_RANGE, E_SHAPE, E_STATE = -3, -2, -4


def calls(p, n, at=FAKE):
    return {
        "fork": lambda: V.vlac_pages_fork(p, at, at, n, check=False),
        "extend": lambda: V.vlac_pages_extend(p, at, n, 1, at, check=False),
        "append": lambda: V.vlac_pages_append(p, 0, at, at, n, 1, FAKE, FAKE, check=False),
        "free": lambda: V.vlac_pages_free(p, at, n, check=False),
        "plan": lambda: V.vlac_attend_plan(p, at, at, n, 1, 4, at, None, check=False),
        "attend": lambda: V.vlac_attend_shared(p, 0, n, 1, 4, FAKE, FAKE, None, check=False),
    }


def test_lists_as_addresses():
    for name, call in calls(pool(), -1).items():
        assert call() == E_RANGE, name
    for name, call in calls(pool(), 0).items():
        assert call() == 0, name
    for name, call in calls(pool(head_dim=96), 1).items():
        assert call() == E_SHAPE, name
    p = pool(data=FAKE + 8)
    assert V.vlac_pages_reset(p, check=False) == E_SHAPE and V.vlac_pages_check(p, check=False) == E_SHAPE
    assert V.vlac_pages_compact(p, FAKE, check=False) == E_SHAPE
    assert V.vlac_pages_import(None, FAKE, 1, 1, pool(), FAKE, check=False) == -1
    assert V.vlac_decode_candidates(None, pool(), FAKE, 1, 1, None, 1, FAKE, FAKE, None, None, check=False) == -1
    assert V.vlac_candidates_workspace_bytes(None, pool(), 1) == 0
    with pytest.raises(V.VlacError):
        V.vlac_pages_free(pool(), FAKE, -1)


def test_no_pool():
    assert V.vlac_pages_free(None, FAKE, 1, check=False) == -1 and V.vlac_pages_compact(None, FAKE, check=False) == -1
    assert V.vlac_pages_reset(None, check=False) == -1


def test_host_tensors_are_refused():
    import torch
    x = torch.zeros(4, dtype=torch.int32)
    for name, call in calls(pool(), 1, at=x).items():
        if name != "attend":
            with pytest.raises(ValueError):
                call()
    with pytest.raises(ValueError):
        V.vlac_attend_shared(pool(), 0, 1, 1, 4, torch.zeros((1, 1, 4, 64), dtype=torch.float16), FAKE, None)
    with pytest.raises(ValueError):
        V.vlac_attend_plan(pool(), FAKE, FAKE, 1, 1, 4, None, torch.zeros(4096, dtype=torch.uint8))
    with pytest.raises(AttributeError):
        pool().nothing
