"""Trees of drafted tokens in plain Python (for the tests): what follows what, which path is accepted, and what keeping it does to
a pool's books."""
import random

from pages_model import PAGE, pages_of


def lineage(parents, t):
    """The nodes from t up to the one that follows the cached sequence, or None: there is no node t."""
    up = []
    while True:
        p = parents[t]
        if p < -1 or p >= t:
            return None
        up.append(t)
        if p == -1:
            return up
        t = p


def places(parents, pos):
    up = [lineage(parents, t) for t in range(len(parents))]
    return [-1 if u is None else pos + len(u) - 1 for u in up]


def tree(rng, tokens, kind="random", there=None):
    """Parents: "random", "chain", "star" (all follow node 0), "roots" (all follow the sequence), "holes" (some are not there)."""
    there = tokens if there is None else there
    par = []
    for t in range(there):
        if t == 0 or kind == "roots":
            par.append(-1)
        elif kind == "chain":
            par.append(t - 1)
        elif kind == "star":
            par.append(0)
        else:
            p = rng.randrange(-1, t) if kind == "holes" else rng.randrange(t)
            par.append(-2 if kind == "holes" and rng.random() < 0.25 else p)
    return par + [-2] * (tokens - there)


def accept(parents, drafted, chosen):
    """-> path, token after it."""
    if parents[0] != -1:
        return [], -1
    path = [0]
    while True:
        more = [t for t in range(1, len(parents)) if parents[t] == path[-1] and parents[t] < t and drafted[t] == chosen[path[-1]] >= 0]
        if not more:
            return path, chosen[path[-1]]
        path.append(more[0])


def keep(pool, seqs, pos, tokens, path, count):
    """pages_model.Pool's books after vlac_pages_keep; -> (entry, from position, to position) of the rows that move."""
    moves, seen, ok = [], set(), []
    for i, (s, p, m) in enumerate(zip(seqs, pos, count)):
        if p < 0:
            continue
        good = pool.seq_ok(s) and s not in seen and p + tokens == pool.len[s] and 0 <= m <= tokens
        seen.add(s)
        mine = path[i][:max(m, 0)]
        good = good and all(0 <= t < tokens for t in mine) and all(a < b for a, b in zip(mine, mine[1:]))
        if good:
            for k, t in enumerate(mine):
                row = pool.table[s]
                if t != k and pool.refs[row[(p + k) // PAGE]] != 1:
                    good = False
        if not good:
            pool.bad = True
            continue
        ok.append((s, p, m))
        moves += [(i, p + t, p + k) for k, t in enumerate(mine) if t != k]
    for s, p, m in ok:
        for j in range(pages_of(p + m), pages_of(p + tokens)):
            pool.refs[pool.table[s][j]] -= 1
            pool.table[s][j] = -1
        pool.len[s] = p + m
    return moves


def some_tree(seed, tokens, kind="random", there=None):
    return tree(random.Random(seed), tokens, kind, there)
