"""A pool of cache pages in plain Python (for the tests): what every entry point of include/vlac.h on pages leaves in
refs, table and len, and which page's values are copied where; and the two tile orders."""
import numpy as np

PAGE = 32
OK, E_RANGE, E_NOMEM = 0, -3, -6


def pages_of(n):
    return -(-n // PAGE)


def k_tile_at(hd):
    """[32, hd]: where feature f of position r stands in a K tile."""
    r, f = np.arange(PAGE)[:, None], np.arange(hd)[None, :]
    return f // 16 * 512 + f // 8 % 2 * 256 + r * 8 + f % 8


def v_tile_at(hd):
    r, f = np.arange(PAGE)[:, None], np.arange(hd)[None, :]
    return f // 32 * 1024 + r // 16 * 512 + r // 4 % 2 * 256 + f % 32 * 8 + r // 8 % 2 * 4 + r % 4


class Pool:
    def __init__(self, n_pages, max_seqs, max_pages):
        self.refs, self.table = [0] * n_pages, [[-1] * max_pages for _ in range(max_seqs)]
        self.len, self.data = [0] * max_seqs, list(range(n_pages))   # data: whose values a page holds
        self.max_pages, self.bad, self.full = max_pages, False, False

    def check(self):
        st = E_NOMEM if self.full else E_RANGE if self.bad else OK
        self.bad = self.full = False
        return st

    def seq_ok(self, s):
        return 0 <= s < len(self.len) and 0 <= self.len[s] <= PAGE * self.max_pages

    def _drop(self, s):
        for j in range(pages_of(self.len[s])):
            self.refs[self.table[s][j]] -= 1
        self.table[s], self.len[s] = [-1] * self.max_pages, 0

    def _take(self, k):
        """The k lowest free pages, or None."""
        free = [p for p, r in enumerate(self.refs) if r == 0][:k]
        return free if len(free) == k else None

    def _entries(self, dst, fits):
        seen, out = set(), []
        for i, d in enumerate(dst):
            ok = self.seq_ok(d) and d not in seen and fits(i, d)
            if 0 <= d < len(self.len):
                seen.add(d)
            self.bad |= not ok
            if ok:
                out.append((i, d))
        return out

    def fork(self, src, dst, deep=False):
        live = self._entries(dst, lambda i, d: self.seq_ok(src[i]) and d not in src)
        saved = ([*self.refs], [[*t] for t in self.table], [*self.len])
        for _, d in live:
            self._drop(d)
        need = [pages_of(self.len[src[i]]) if deep else int(self.len[src[i]] % PAGE != 0) for i, _ in live]
        fresh = self._take(sum(need))
        if fresh is None:
            self.refs, self.table, self.len = saved
            self.full = True
            return
        before = [*self.data]
        for (i, d), k in zip(live, need):
            s = src[i]
            n = pages_of(self.len[s])
            for j in range(n):
                p = self.table[s][j]
                if j >= n - k:
                    p = fresh.pop(0)
                    self.data[p] = before[self.table[s][j]]
                self.refs[p] += 1
                self.table[d][j] = p
            self.len[d] = self.len[s]

    def extend(self, seqs, tokens):
        live = self._entries(seqs, lambda i, s: self.len[s] + tokens <= PAGE * self.max_pages)
        pos = [-1] * len(seqs)
        need = [pages_of(self.len[s] + tokens) - pages_of(self.len[s]) for _, s in live]
        fresh = self._take(sum(need))
        if fresh is None:
            self.full = True
            return pos
        for (i, s), k in zip(live, need):
            pos[i] = self.len[s]
            for j in range(k):
                p = fresh.pop(0)
                self.table[s][pages_of(self.len[s]) + j] = p
                self.refs[p] = 1
            self.len[s] += tokens
        return pos

    def free(self, seqs):
        for s in seqs:
            if self.seq_ok(s):
                self._drop(s)
            else:
                self.bad = True

    def compact(self):
        live = sum(r > 0 for r in self.refs)
        holes = [p for p in range(live) if self.refs[p] == 0]
        to = {}
        for p in range(live, len(self.refs)):
            if self.refs[p] > 0:
                d = to[p] = holes.pop(0)
                self.data[d] = self.data[p]
                self.refs[d], self.refs[p] = self.refs[p], 0
        self.table = [[to.get(p, p) for p in t] for t in self.table]
        return live
