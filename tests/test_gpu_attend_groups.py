"""Many groups for few kv heads: an XCD's runs of work items, blocks of few whole entries, and where neither applies."""
import random

import pytest

from test_gpu_attend import Cache, definition, run
from test_gpu_attend import DEV

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("hq,hkv,hd,operand", [(2, 1, 64, 1), (12, 2, 128, 0), (8, 4, 64, 0), (16, 8, 64, 1), (6, 3, 128, 1),
                                               (40, 40, 64, 1)])
@pytest.mark.parametrize("groups,most,T", [(1, 40, 1), (7, 3, 1), (9, 9, 2), (65, 5, 1), (130, 2, 1), (33, 1, 17)])
def test_many_groups(hq, hkv, hd, operand, groups, most, T):
    """Groups of 1 to `most` entries over stems of 0 to 5 pages; the last group is the largest, so that runs are uneven."""
    import torch
    rng = random.Random(1000 * groups + hkv)
    cache = Cache(hkv, hd, operand, groups)
    seqs, pos, label = [], [], []
    for g in range(groups):
        first = cache.sequence(rng.randrange(0, 5 * 32) + T)
        full, length = cache.seqs[first][0], cache.seqs[first][1]
        for _ in range(most if g == groups - 1 else rng.randrange(1, most + 1)):
            shared = full[:rng.randrange(0, (length - T) // 32 + 1)]
            s = cache.sequence(max(32 * len(shared) + T, length - rng.randrange(0, 2)), shared)
            seqs.append(s)
            pos.append(cache.seqs[s][1] - T)
            label.append(g % 2)
    p = cache.pool()
    q = torch.randn((len(seqs), T, hq, hd), generator=cache.g, device=DEV).to(cache.dt)
    out = run(p, cache, seqs, pos, q, label)
    want, tol = definition(cache, seqs, pos, q)
    assert bool(((out.double() - want).abs() <= tol).all())
