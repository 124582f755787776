"""Lists of every length that the planning kernels treat differently (compared pair by pair up to 256 entries, by marks beyond;
several rounds of threads), full of sequences listed twice and of destinations that are sources."""
import random

import pytest

from test_gpu_pages import Both

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n", [1, 2, 31, 32, 33, 63, 100, 255, 256, 257, 600, 1025, 2100])
def test_repeated_entries_count_once(n):
    rng = random.Random(n)
    seqs = 3 * n + 2
    b = Both(6 * n + 8, seqs, 3)
    b.extend([rng.randrange(seqs) for _ in range(n)], 33)
    b.same("extend")
    b.extend([rng.choice([rng.randrange(seqs), rng.randrange(max(n // 4, 1))]) for _ in range(n)], 20)
    b.same("extend again")
    # the last entry repeats the first, the one before it is a source
    src = [rng.randrange(seqs) for _ in range(n)]
    dst = [rng.randrange(seqs) for _ in range(n)]
    dst[-1] = dst[0]
    if n > 2:
        dst[-2] = src[0]
    b.fork(src, dst)
    b.same("fork")
    b.fork(dst, [s for s in src], True)
    b.same("deep")
    b.free(dst)
    b.same("free")
    b.compact()
    b.same("compact")
