"""The operators by which a program checks a tree of drafted tokens against a paged KV cache in one
pass, as cases that can be timed and checked: keys and values appended with the norm of every head and
the rotation of its position applied on the way, attention of the tree's nodes over the cache and their
ancestors, the choice of a token under penalties, biases and a grammar's mask, and the accepted path
kept in the cache.

A page holds K and V of 32 positions for all layers, [layer][K, V][kv head][32 * head_dim], a
head's 32 positions in the order in which the matrix cores take them:
  K  [head_dim / 16][2][32 positions][8]          feature 16 a + 8 g + e of position r at [a][g][r][e]
  V  [head_dim / 32][2][2][32 features][2][4]     feature 32 b + f of position 16 t + 8 i + 4 g + e at [b][t][g][f][i][e]
table [sequences, pages per sequence] names a sequence's pages (-1 behind its last), len its
positions, refs how many table entries name a page.

The tree of an entry has `nodes` places: parents[i, t] < t is the node that t follows, -1 the
cached sequence, -2 says that there is no node (trees of a batch differ in size).  Node t has the slot
pos[i] + t in the cache until the path is kept, and the place pos[i] + (its ancestors) in the text.

`run` is one pass as a program makes it, in elementary torch operations or (own) by the library.
Sizes are functions of the case, values, trees and tokens come from the seed."""
import math
import random

import torch

own = False

DEV = "cuda:0"
PAGE = 32
# query heads, kv heads, head_dim: the decoder shapes of this repository, and two generic layouts
HEADS = {"tiny": (4, 4, 64), "7b": (32, 32, 128), "gqa": (12, 2, 128), "g4": (16, 4, 64), "mqa": (8, 1, 128)}
DTYPE = {"bf16": torch.bfloat16, "f16": torch.float16}
EPS = 1e-6


def listed():
    return [
        # one token of two sequences of the smoke shape, a part of every head rotated: launches and latency
        dict(name="append_tiny", kind="append", heads="tiny", dtype="f16", layers=2, groups=2, cands=1, prefix=80, nodes=1,
             layout="pairs", dims=32, base=10000.0, factor=1.0, original=0, norm=False),
        # the drafts of 8 sequences of the large decoder, several layers
        dict(name="append_7b_drafts", kind="append", heads="7b", dtype="f16", layers=4, groups=8, cands=1, prefix=303, nodes=31,
             layout="half", dims=128, base=10000.0, factor=1.0, original=0, norm=False),
        # a long piece of 4 prompts at far positions, heads normed, wavelengths scaled by bands
        dict(name="append_prompt_gqa", kind="append", heads="gqa", dtype="bf16", layers=2, groups=4, cands=1, prefix=33000, nodes=1057,
             layout="half", dims=128, base=500000.0, factor=8.0, original=8192, norm=True),
        # a small tree behind a short sequence of the smoke shape: latency
        dict(name="tree_tiny", kind="tree", heads="tiny", dtype="f16", layers=2, groups=1, cands=1, prefix=80, nodes=7),
        # trees of 32 environments, grouped queries
        dict(name="tree_gqa_32", kind="tree", heads="gqa", dtype="bf16", layers=4, groups=32, cands=1, prefix=304, nodes=24),
        # trees of 8 candidates of one two-view observation
        dict(name="tree_7b_cands", kind="tree", heads="7b", dtype="f16", layers=2, groups=1, cands=8, prefix=1057, nodes=16),
        # large trees behind two long histories, odd length
        dict(name="tree_long", kind="tree", heads="7b", dtype="f16", layers=2, groups=2, cands=1, prefix=32801, nodes=64),
        # the next token of one sequence, only the bins of an action allowed
        dict(name="choose_one", kind="choose", entries=1, nodes=1, vocab=32000, history=300, mask="few", repetition=1.2,
             presence=0.0, frequency=0.0, bias=False),
        # every node of 8 trees: the history and the path above the node count
        dict(name="choose_tree", kind="choose", entries=8, nodes=32, vocab=32000, history=1057, mask="most", repetition=1.1,
             presence=0.3, frequency=0.2, bias=True),
        # a batch with long histories over a large vocabulary of odd size
        dict(name="choose_wide", kind="choose", entries=96, nodes=1, vocab=150001, history=4000, mask="most", repetition=1.0,
             presence=0.5, frequency=0.1, bias=True),
        # the accepted paths of two small trees of the smoke shape, and of 8 of the large decoder, all layers
        dict(name="settle_tiny", kind="settle", heads="tiny", dtype="f16", layers=2, groups=2, cands=1, prefix=80, nodes=7),
        dict(name="settle_7b", kind="settle", heads="7b", dtype="f16", layers=32, groups=8, cands=1, prefix=303, nodes=31),
    ]


def draw(rng):
    def log_int(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    top = {}
    for c in listed():
        w = work(c)
        for k in w:
            top[k] = max(top.get(k, 0), w[k])
    while True:
        kind = rng.choice(["append", "tree", "tree", "choose", "settle"])
        c = dict(kind=kind)
        if kind == "choose":
            c.update(entries=log_int(1, 256), nodes=1 if rng.random() < 0.5 else log_int(2, 100), vocab=log_int(100, 200000),
                     history=log_int(1, 5000), mask=rng.choice(["none", "few", "most"]), repetition=rng.choice([1.0, 1.1, 1.3]),
                     presence=rng.choice([0.0, 0.4]), frequency=rng.choice([0.0, 0.25]), bias=rng.random() < 0.5)
        else:
            heads = rng.choice(["tiny", "7b", "7b", "gqa", "gqa", "g4", "mqa"])
            c.update(heads=heads, dtype=rng.choice(["f16", "bf16"]), layers=rng.randint(1, 32 if kind == "settle" else 4),
                     groups=log_int(1, 32), cands=1, prefix=log_int(1, 33000 if kind == "tree" else 1100), nodes=log_int(1, 200))
            if kind == "append":
                hd = HEADS[heads][2]
                c.update(nodes=log_int(1, 1100), layout=rng.choice(["half", "pairs"]),
                         dims=hd if rng.random() < 0.5 else 2 * rng.randint(1, hd // 2), base=rng.choice([10000.0, 500000.0]),
                         factor=rng.choice([1.0, 4.0, 8.0]), original=rng.choice([0, 4096, 8192]), norm=rng.random() < 0.5)
            if kind == "tree":
                c["cands"] = log_int(1, 16)
        w = work(c)
        if w["flops"] <= top["flops"] and w["bytes"] <= top["bytes"] and _pool_bytes(c) <= 4e9 and _plain_bytes(c) <= 8e9:
            return c


# ------------------------------------------------------------------------------------------
# sizes, from the case alone
# ------------------------------------------------------------------------------------------
def _up(x):
    return -(-x // PAGE)


def _prefixes(c):
    """Cached positions of every group: the first has the most."""
    return [max(1, c["prefix"] - 11 * g % 37 - (g % 5 == 4) * (c["prefix"] // 3)) for g in range(c["groups"])]


def _entries(c):
    """(group, cached positions) of every entry, group by group; candidates of a group share its full pages."""
    return [(g, p + 5 * k % 23) for g, p in enumerate(_prefixes(c)) for k in range(c["cands"])]


def _sizes(c, n):
    """Nodes of every tree: the first is whole."""
    T = c["nodes"]
    return [T - 5 * i % (T // 3 + 1) for i in range(n)]


def _accepted(c, n):
    """Nodes on the accepted path of every entry."""
    return [1 + (3 * i + 4) % min(m, 7) for i, m in enumerate(_sizes(c, n))]


def _page_elems(c):
    _, hkv, hd = HEADS[c["heads"]]
    return c["layers"] * 2 * hkv * PAGE * hd


def _page_counts(c):
    """-> pages in the pool, pages per sequence."""
    ent, pre = _entries(c), _prefixes(c)
    most = max(p for _, p in ent) + c["nodes"]
    held = sum(p // PAGE for p in pre) + sum(_up(p + c["nodes"]) - pre[g] // PAGE for g, p in ent)
    return held + 5, _up(most) + 1


def _pool_bytes(c):
    return 0 if c["kind"] == "choose" else _page_counts(c)[0] * _page_elems(c) * 2


def _plain_bytes(c):
    """The plain form's arrays in 32 bits."""
    if c["kind"] == "choose":
        return 24 * c["entries"] * c["nodes"] * c["vocab"]
    hq, hkv, hd = HEADS[c["heads"]]
    n, most = len(_entries(c)), PAGE * _page_counts(c)[1]
    if c["kind"] == "tree":
        return 4 * n * most * (2 * c["nodes"] * hq + 4 * hkv * hd)
    return 32 * n * c["nodes"] * (hq + 2 * hkv) * hd * (c["layers"] if c["kind"] == "settle" else 1)


def work(case):
    c = case
    if c["kind"] == "choose":
        rows, n = c["entries"] * c["nodes"], c["entries"]
        b = 8 * rows * c["vocab"] + 4 * n * c["history"] + 12 * rows + (4 * c["vocab"] if c["bias"] else 0)
        return {"bytes": b + (0 if c["mask"] == "none" else rows * c["vocab"] // 8), "flops": 0}
    hq, hkv, hd = HEADS[c["heads"]]
    ent, L = _entries(c), c["layers"]
    n, sizes = len(ent), _sizes(c, len(ent))
    row = hkv * hd * 2 * 2                                    # K and V of one position and layer
    if c["kind"] == "append":
        rows = L * n * c["nodes"]
        return {"bytes": rows * 2 * (hq * hd * 2 + row), "flops": rows * (hq + hkv) * (3 * c["dims"] + (4 * hd if c["norm"] else 0))}
    if c["kind"] == "settle":
        return {"bytes": 2 * L * row * sum(a - 1 for a in _accepted(c, n)) + 12 * sum(sizes) + 64 * n, "flops": 0}
    pre = _prefixes(c)
    read = sum(p // PAGE * PAGE for p in pre) + sum(p - pre[g] // PAGE * PAGE + m for (g, p), m in zip(ent, sizes))
    return {"bytes": L * (read * row + 2 * sum(sizes) * hq * hd * 2) + 4 * n * c["nodes"],
            "flops": L * 4 * hd * hq * sum(m * (p + 1) for (_, p), m in zip(ent, sizes))}


# ------------------------------------------------------------------------------------------
# inputs, from the seed alone
# ------------------------------------------------------------------------------------------
def _gen(seed, *tags):
    g = torch.Generator(device=DEV)
    s = int(seed) & 0xFFFFFFFF
    for t in tags:
        s = (s * 1000003 + int(t) + 1) & 0x7FFFFFFFFFFFFFFF
    g.manual_seed(s)
    return g


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def _k_tiles(x):
    """[..., 32, hd] -> [..., 32 * hd] in the order of a K tile."""
    *lead, _, hd = x.shape
    return x.reshape(*lead, PAGE, hd // 16, 2, 8).movedim(-4, -2).reshape(*lead, PAGE * hd)


def _v_tiles(x):
    *lead, _, hd = x.shape
    y = x.reshape(*lead, 2, 2, 2, 4, hd // 32, 32)           # t, i, g, e, b, f
    n = len(lead)
    return y.permute(*range(n), n + 4, n, n + 2, n + 5, n + 1, n + 3).reshape(*lead, PAGE * hd)


def _trees(c, n, seed, vocab=32000):
    """-> parents, drafted tokens, chosen tokens, all [n][nodes]: random trees, on one path of which the drafts are what was
    chosen.  The root is a token that is known (chosen in the pass before)."""
    rng = random.Random(int(seed) * 7919 + 5)
    T = c["nodes"]
    parents, drafted, chosen = [], [], []
    for m, a in zip(_sizes(c, n), _accepted(c, n)):
        path = [0] + sorted(rng.sample(range(1, m), a - 1))
        par = [-1] + [int(t * rng.random()) for t in range(1, m)]
        for u, t in zip(path, path[1:]):
            par[t] = u
        tok = [rng.randrange(vocab - 1) for _ in range(m)]
        for u, t in zip(path, path[1:]):                      # (a later twin of an accepted draft is never taken)
            for s in range(1, t):
                if par[s] == u and tok[s] == tok[t]:
                    tok[s] = (tok[t] + 1) % (vocab - 1)
        ch = [rng.randrange(vocab - 1) for _ in range(m)]
        for u, t in zip(path, path[1:]):
            ch[u] = tok[t]
        ch[path[-1]] = vocab - 1                              # (nobody drafted that)
        parents.append(par + [-2] * (T - m))
        drafted.append(tok + [0] * (T - m))
        chosen.append(ch + [0] * (T - m))
    return _i32(parents), _i32(drafted), _i32(chosen)


def _choose_inputs(c, seed):
    n, T, vocab, H = c["entries"], c["nodes"], c["vocab"], c["history"]
    rows = n * T
    s = {"c": c, "logits": 3.0 * torch.randn((rows, vocab), generator=_gen(seed, 1), device=DEV)}
    # few tokens make up most of a text
    u = torch.rand((n, H), generator=_gen(seed, 2), device=DEV, dtype=torch.float64)
    s["history"] = (u.pow(3) * vocab).to(torch.int32).clamp(max=vocab - 1)
    s["history_len"] = _i32([max(0, H - 37 * i % (H // 2 + 1)) for i in range(n)])
    s["bias"] = None
    if c["bias"]:
        b = torch.randn(vocab, generator=_gen(seed, 3), device=DEV)
        s["bias"] = torch.where(torch.rand(vocab, generator=_gen(seed, 4), device=DEV) < 0.05, 4.0 * b, 0.0)
    s["allowed"] = None
    if c["mask"] != "none":
        words = -(-vocab // 32)
        x = torch.randint(-2 ** 31, 2 ** 31, (rows, words), generator=_gen(seed, 5), device=DEV)
        if c["mask"] == "most":
            x |= torch.randint(-2 ** 31, 2 ** 31, (rows, words), generator=_gen(seed, 6), device=DEV)
        else:                                                 # bins at the end of the vocabulary
            x[:, :max(0, words - 9)] = 0
        s["allowed"] = x.to(torch.int32)
    s["parents"] = s["drafted"] = None
    if T > 1:
        s["parents"], s["drafted"], _ = _trees(c, n, seed, vocab)
    s["out"] = torch.zeros((rows, vocab), device=DEV)
    s["token"] = torch.zeros(rows, dtype=torch.int32, device=DEV)
    return s


def _inputs(c, seed):
    """Everything that a program has in hand, as plain tensors."""
    if c["kind"] == "choose":
        return _choose_inputs(c, seed)
    hq, hkv, hd = HEADS[c["heads"]]
    dt, T, L, ent = DTYPE[c["dtype"]], c["nodes"], c["layers"], _entries(c)
    n, pre = len(ent), _prefixes(c)
    n_pages, max_pages = _page_counts(c)
    s = {"c": c, "dt": dt}
    order = iter(torch.randperm(n_pages, generator=_gen(seed, 1), device=DEV).tolist())    # where a long run left them
    stems = [[next(order) for _ in range(p // PAGE)] for p in pre]
    table, refs, fresh = [[-1] * max_pages for _ in range(n + 2)], [0] * n_pages, [(p, PAGE) for st in stems for p in st]
    for i, (g, p) in enumerate(ent):
        mine = list(stems[g])
        while len(mine) < _up(p + T):
            q = next(order)
            filled = p + (0 if c["kind"] == "append" else T) - PAGE * len(mine)
            fresh.append((q, max(0, min(PAGE, filled))))
            mine.append(q)
        table[i][:len(mine)] = mine
        for q in mine:
            refs[q] += 1
    # positions that no token was ever written to hold NaN patterns, as fresh memory may (append: zeros)
    pool = torch.full((n_pages, L, 2, hkv, PAGE * hd), 0 if c["kind"] == "append" else -1, dtype=torch.int16, device=DEV)
    pages, filled = torch.tensor([p for p, _ in fresh], device=DEV), torch.tensor([f for _, f in fresh], device=DEV)
    g2, step = _gen(seed, 2), max(1, int(2e8) // (2 * hkv * PAGE * hd))          # (in pieces: the 32-bit draws are large)
    for l in range(L):
        for a in range(0, len(fresh), step):
            x = torch.randn((len(pages[a:a + step]), 2, hkv, PAGE, hd), generator=g2, device=DEV).to(dt).view(torch.int16)
            hole = torch.arange(PAGE, device=DEV)[None, :] >= filled[a:a + step, None]
            x = x.masked_fill_(hole[:, None, None, :, None], 0 if c["kind"] == "append" else -1)
            pool[pages[a:a + step], l] = torch.stack([_k_tiles(x[:, 0]), _v_tiles(x[:, 1])], 1)
    s["pool"], s["table"], s["refs"] = pool, _i32(table), _i32(refs)
    s["len"] = _i32([p + T for _, p in ent] + [0, 0])
    s["seqs"], s["pos"], s["group"] = _i32(list(range(n))), _i32([p for _, p in ent]), _i32([g for g, _ in ent])
    s["parents"], s["drafted"], s["chosen"] = _trees(c, n, seed)
    if c["kind"] == "append":
        # a joint projection's rows: query heads, key heads, value heads
        s["qkv"] = torch.randn((L, n, T, hq + 2 * hkv, hd), generator=_gen(seed, 3), device=DEV).to(dt)
        s["q_gain"], s["k_gain"] = [(1 + 0.1 * torch.randn(hd, generator=_gen(seed, 4 + k), device=DEV)).bfloat16() for k in (0, 1)]
        s["out"] = torch.zeros((L, n, T, hq, hd), dtype=dt, device=DEV)
    if c["kind"] == "tree":
        # sharp enough that a few dozen positions carry most of the weight
        s["q"] = (2.5 * torch.randn((L, n, T, hq, hd), generator=_gen(seed, 3), device=DEV)).to(dt)
        s["out"] = torch.zeros((L, n, T, hq, hd), dtype=dt, device=DEV)
    if c["kind"] == "settle":
        s["path"], s["count"], s["token"] = torch.zeros_like(s["parents"]), torch.zeros_like(s["pos"]), torch.zeros_like(s["pos"])
        s["table0"], s["refs0"], s["len0"] = s["table"].clone(), s["refs"].clone(), s["len"].clone()
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    if own:
        import paper_2502_02175_amd as V
        c = case
        s["V"] = V
        u8 = dict(dtype=torch.uint8, device=DEV)
        if c["kind"] == "choose":
            s["ws"] = torch.empty(V.vlac_choose_workspace_bytes(c["entries"] * c["nodes"], c["vocab"]), **u8)
            s["rules"] = V.token_rules(repetition=c["repetition"], presence=c["presence"], frequency=c["frequency"], bias=s["bias"],
                                       allowed=s["allowed"], history=s["history"], history_len=s["history_len"],
                                       parents=s["parents"], drafted=s["drafted"])
            return s
        hq, hkv, hd = HEADS[c["heads"]]
        s["pages"] = V.pages(c["layers"], hkv, hd, V.OPERAND_F16 if c["dtype"] == "f16" else V.OPERAND_BF16,
                             s["pool"], s["refs"], s["table"], s["len"])
        if c["kind"] == "append":
            s["rot"] = V.rotary(c["dims"], V.ROTARY_HALF if c["layout"] == "half" else V.ROTARY_PAIRS, c["base"], c["factor"],
                                c["original"], 1.0, 4.0)
            # the places of the tree's nodes, or of a plain piece of text
            s["places"] = None if c["nodes"] > 200 else _places(s).to(torch.int32)
        if c["kind"] == "tree":
            s["ws"] = torch.empty(V.vlac_attend_tree_workspace_bytes(s["pages"], len(_entries(c)), c["nodes"], hq), **u8)
            s["places"] = torch.zeros_like(s["parents"])
    elif case["kind"] == "append":
        s["places"] = None if case["nodes"] > 200 else _places(s).to(torch.int32)
    return s


# ------------------------------------------------------------------------------------------
# one pass
# ------------------------------------------------------------------------------------------
def run(state):
    s, kind = state, state["c"]["kind"]
    if kind == "append":
        (_own_append if own else _append)(s)
        return {"q": s["out"], "pool": s["pool"].view(s["dt"])}
    if kind == "tree":
        (_own_tree if own else _tree)(s)
        return {"out": s["out"], "places": s["places"]}
    if kind == "choose":
        (_own_choose if own else _choose)(s)
        return {"logits": s["out"], "token": s["token"]}
    s["table"].copy_(s["table0"])                             # (the pool's books as they were before the last pass)
    s["refs"].copy_(s["refs0"])
    s["len"].copy_(s["len0"])
    (_own_settle if own else _settle)(s)
    return {k: s[k] for k in ("path", "count", "token", "pool", "table", "refs", "len")}


def _own_append(s):
    V, c = s["V"], s["c"]
    hq, hkv, _ = HEADS[c["heads"]]
    n, gains = s["seqs"].numel(), (s["q_gain"], s["k_gain"], EPS) if c["norm"] else (None, None, EPS)
    for l in range(c["layers"]):
        q, k, v = s["qkv"][l].split((hq, hkv, hkv), 2)
        V.vlac_pages_append_rotated(s["pages"], l, s["seqs"], s["pos"], n, c["nodes"], s["rot"], s["places"], hq, q, k, v,
                                    s["out"][l], *gains)


def _own_tree(s):
    V, c = s["V"], s["c"]
    n, T, hq = s["seqs"].numel(), c["nodes"], HEADS[c["heads"]][0]
    V.vlac_attend_tree_plan(s["pages"], s["seqs"], s["pos"], n, T, hq, s["group"], s["parents"], s["places"], s["ws"])
    for l in range(c["layers"]):
        V.vlac_attend_tree(s["pages"], l, n, T, hq, s["q"][l], s["out"][l], s["ws"])


def _own_choose(s):
    s["V"].vlac_choose_tokens(s["logits"], s["rules"], s["out"], s["token"], s["ws"])


def _own_settle(s):
    V, n, T = s["V"], s["seqs"].numel(), s["c"]["nodes"]
    V.vlac_tree_accept(s["parents"], s["drafted"], s["chosen"], n, T, s["path"], s["count"], s["token"])
    V.vlac_pages_keep(s["pages"], s["seqs"], s["pos"], n, T, s["path"], s["count"])


# the plain forms ---------------------------------------------------------------------------
def _lineage(parents):
    """[n, T] -> [n, T, T]: whether u is t or above it (by doubling), in 32 bits."""
    n, T = parents.shape
    at = torch.arange(T, device=DEV)
    x = ((at[None, None, :] == parents[:, :, None]) | (at[None, None, :] == at[None, :, None])).float()
    x = torch.where((parents >= -1)[:, :, None], x, 0.0)
    for _ in range(max(1, (T - 1).bit_length())):
        x = (torch.matmul(x, x) > 0).float()
    return x


def _places(s):
    """Where every node stands in the text (-1: no node)."""
    depth = _lineage(s["parents"]).sum(-1).to(torch.int64) - 1
    return torch.where(s["parents"] >= -1, s["pos"].long()[:, None] + depth, -1)


def _turns(c):
    """Radians per position of every rotated pair, in 64 bits."""
    half = c["dims"] // 2
    w = c["base"] ** (-torch.arange(half, device=DEV, dtype=torch.float64) * 2 / c["dims"])
    if c["original"] == 0:
        return w / c["factor"]
    keep = ((c["original"] * w / (2 * math.pi) - 1.0) / (4.0 - 1.0)).clamp(0.0, 1.0)
    return w * (keep + (1 - keep) / c["factor"])


def _normed(x, gain):
    return x * torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS) * gain.float()


def _rotated(x, cos, sin, c):
    """x [n, T, heads, hd] in 32 bits."""
    d = c["dims"]
    y, rest = x[..., :d], x[..., d:]
    if c["layout"] == "half":
        a, b = y[..., :d // 2], y[..., d // 2:]
        return torch.cat([a * cos - b * sin, b * cos + a * sin, rest], -1)
    a, b = y[..., 0::2], y[..., 1::2]
    return torch.cat([torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2), rest], -1)


def _append(s):
    c = s["c"]
    hq, hkv, hd = HEADS[c["heads"]]
    T = c["nodes"]
    at = s["pos"].long()[:, None] + torch.arange(T, device=DEV)[None, :]
    places = at if s["places"] is None else s["places"].long()
    there = (places >= 0)[:, :, None, None]
    angle = places.double()[:, :, None] * _turns(c)
    cos, sin = (f(angle).float()[:, :, None, :] for f in (torch.cos, torch.sin))
    page = s["table"].long()[s["seqs"].long()[:, None], at // PAGE].reshape(-1)
    r = (at % PAGE).reshape(-1)
    for l in range(c["layers"]):
        x = s["qkv"][l].float()
        q, k, v = x.split((hq, hkv, hkv), 2)
        if c["norm"]:
            q, k = _normed(q, s["q_gain"]), _normed(k, s["k_gain"])
        q, k = (torch.where(there, _rotated(y, cos, sin, c), 0.0).to(s["dt"]) for y in (q, k))
        v = torch.where(there, v, 0.0).to(s["dt"])
        s["out"][l] = q
        kv = s["pool"][:, l, 0].view(-1, hkv, hd // 16, 2, PAGE, 8)
        kv[page, :, :, :, r] = k.view(torch.int16).reshape(-1, hkv, hd // 16, 2, 8)
        vv = s["pool"][:, l, 1].view(-1, hkv, hd // 32, 2, 2, 32, 2, 4)
        vv[page, :, :, r // 16, r // 4 % 2, :, r // 8 % 2, r % 4] = v.view(torch.int16).reshape(-1, hkv, hd // 32, 32)


def _gather(s, layer, which, pages):
    """[n, j] page indices -> K or V rows in 32 bits, [n, hkv, 32 j, hd]."""
    _, hkv, hd = HEADS[s["c"]["heads"]]
    n, j = pages.shape
    x = s["pool"][pages, layer, which].view(s["dt"]).float()
    if which == 0:
        y = x.view(n, j, hkv, hd // 16, 2, PAGE, 8).permute(0, 2, 1, 5, 3, 4, 6)
    else:
        y = x.view(n, j, hkv, hd // 32, 2, 2, 32, 2, 4).permute(0, 2, 1, 4, 7, 5, 8, 3, 6)
    return y.reshape(n, hkv, j * PAGE, hd)


def _tree(s):
    c = s["c"]
    hq, hkv, hd = HEADS[c["heads"]]
    n, T, grp = s["seqs"].numel(), c["nodes"], hq // hkv
    line = _lineage(s["parents"])
    there = s["parents"] >= -1
    s["places"] = _places(s).to(torch.int32)
    pages = s["table"].long()[s["seqs"].long()][:, :_up(max(p for _, p in _entries(c)) + T)].clamp(min=0)
    at = torch.arange(PAGE * pages.shape[1], device=DEV)
    node = at[None, :] - s["pos"].long()[:, None]              # [n, S]: which node a position holds
    seen = (node < 0)[:, None, :] | ((node >= 0) & (node < T))[:, None, :] & (
        torch.gather(line, 2, node.clamp(0, T - 1)[:, None, :].expand(n, T, -1)) > 0)
    seen = (seen & there[:, :, None])[:, None, :, None, :]     # [n, 1, T, 1, S]
    held = (node < T)[:, None, :, None]
    for l in range(c["layers"]):
        q = s["q"][l].float().view(n, T, hkv, grp, hd).permute(0, 2, 1, 3, 4).reshape(n, hkv, T * grp, hd)
        k, v = (torch.where(held, _gather(s, l, w, pages), 0.0) for w in (0, 1))
        x = torch.matmul(q, k.transpose(2, 3).contiguous()) * (1.0 / math.sqrt(hd))
        x = torch.where(seen, x.view(n, hkv, T, grp, -1), -math.inf)
        top = x.amax(-1, keepdim=True)
        w = torch.exp(x - torch.where(top == -math.inf, 0.0, top))
        den = w.sum(-1, keepdim=True)
        y = torch.matmul(w.view(n, hkv, T * grp, -1), v).view(n, hkv, T, grp, hd)
        y = torch.where(den > 0, y / den, 0.0)
        s["out"][l] = y.permute(0, 2, 1, 3, 4).reshape(n, T, hq, hd).to(s["dt"])


def _choose(s):
    c = s["c"]
    n, T, vocab, H = c["entries"], c["nodes"], c["vocab"], c["history"]
    told = (torch.arange(H, device=DEV)[None, :] < s["history_len"][:, None]).float()
    counts = torch.zeros((n, vocab), device=DEV).scatter_add_(1, s["history"].long(), told)
    counts = counts[:, None, :].expand(n, T, vocab)
    if T > 1:
        line = _lineage(s["parents"])                         # (a node's own token and those above it)
        counts = counts.scatter_add(2, s["drafted"].long()[:, None, :].expand(n, T, T), line)
    counts = counts.reshape(n * T, vocab)
    x = s["logits"]
    hit = counts > 0
    x = torch.where(hit, torch.where(x > 0, x / c["repetition"], x * c["repetition"]), x)
    x = torch.where(hit, x - c["presence"], x)
    x = x - c["frequency"] * counts
    if s["bias"] is not None:
        x = x + s["bias"]
    if s["allowed"] is not None:
        bits = s["allowed"][:, :, None] >> torch.arange(32, device=DEV) & 1
        x = torch.where(bits.reshape(n * T, -1)[:, :vocab] != 0, x, -math.inf)
    s["out"].copy_(x)
    top = x.amax(1, keepdim=True)
    first = torch.where(x == top, torch.arange(vocab, device=DEV, dtype=torch.int32), vocab).amin(1)
    s["token"].copy_(torch.where(top[:, 0] == -math.inf, -1, first))


def _settle(s):
    c = s["c"]
    _, hkv, hd = HEADS[c["heads"]]
    n, T = s["parents"].shape
    parents, drafted = s["parents"].long(), s["drafted"]
    line, at = _lineage(s["parents"]), torch.arange(T, device=DEV)
    follows = drafted == torch.gather(s["chosen"], 1, parents.clamp(min=0))
    twin = (parents[:, :, None] == parents[:, None, :]) & (drafted[:, :, None] == drafted[:, None, :]) & (at[None, :] < at[:, None])
    good = (parents >= 0) & follows & ~twin.any(2)
    good[:, 0] = parents[:, 0] >= -1
    took = (torch.matmul(line, (~good).float()[:, :, None])[:, :, 0] == 0) & (line[:, :, 0] > 0)
    count = took.sum(1)
    path = torch.sort(torch.where(took, at, T), 1).values
    s["path"].copy_(torch.where(path < T, path, -1))
    s["count"].copy_(count)
    last = torch.gather(path, 1, (count - 1).clamp(min=0)[:, None]).clamp(max=T - 1)
    s["token"].copy_(torch.where(count > 0, torch.gather(s["chosen"], 1, last)[:, 0], -1))
    # the rows of the path, one behind the other
    seqs, pos = s["seqs"].long(), s["pos"].long()
    which, k = torch.nonzero(path < T, as_tuple=True)
    rows = [pos[which] + path[which, k], pos[which] + k]
    (p0, r0), (p1, r1) = [(s["table"].long()[seqs[which], x // PAGE], x % PAGE) for x in rows]
    kt = s["pool"][:, :, 0].view(-1, c["layers"], hkv, hd // 16, 2, PAGE, 8)
    vt = s["pool"][:, :, 1].view(-1, c["layers"], hkv, hd // 32, 2, 2, 32, 2, 4)
    kt[p1, :, :, :, :, r1] = kt[p0, :, :, :, :, r0]
    vt[p1, :, :, :, r1 // 16, r1 // 4 % 2, :, r1 // 8 % 2, r1 % 4] = vt[p0, :, :, :, r0 // 16, r0 // 4 % 2, :, r0 // 8 % 2, r0 % 4]
    # what lies behind the path is released
    length = pos + count
    col = torch.arange(s["table"].shape[1], device=DEV)
    mine = s["table"][seqs]
    gone = (col[None, :] >= ((length + PAGE - 1) // PAGE)[:, None]) & (mine >= 0)
    s["refs"].index_add_(0, mine.clamp(min=0).reshape(-1), -gone.to(torch.int32).reshape(-1))
    s["table"][seqs] = torch.where(gone, -1, mine)
    s["len"][seqs] = length.to(torch.int32)


# ------------------------------------------------------------------------------------------
# the definition, in 64 bits and one entry at a time
# ------------------------------------------------------------------------------------------
def _tile_at(hd):
    """[32, hd]: where a feature of a position stands in a K and in a V tile."""
    f, r = torch.arange(hd, device=DEV)[None, :], torch.arange(PAGE, device=DEV)[:, None]
    return (f // 16 * 512 + f // 8 % 2 * 256 + f % 8 + r * 8,
            f // 32 * 1024 + f % 32 * 8 + r // 16 * 512 + r // 4 % 2 * 256 + r // 8 % 2 * 4 + r % 4)


def _above(par, t):
    """t and the nodes above it."""
    up = []
    while t >= 0:
        up.append(t)
        t = par[t]
    return up


def _exact_append(s):
    c = s["c"]
    hq, hkv, hd = HEADS[c["heads"]]
    T, d = c["nodes"], c["dims"]
    k_at, v_at = _tile_at(hd)
    pool = s["pool"].view(s["dt"]).double()
    out = torch.zeros(s["out"].shape, dtype=torch.float64, device=DEV)
    rates = []
    for f in range(d // 2):
        w = c["base"] ** (-2.0 * f / d)
        if c["original"]:
            r = c["original"] * w / (2 * math.pi)
            w = w if r > 4 else w / c["factor"] if r < 1 else (r - 1) / 3 * w + (4 - r) / 3 * w / c["factor"]
        else:
            w /= c["factor"]
        rates.append(w)
    rates = torch.tensor(rates, dtype=torch.float64, device=DEV)
    first = torch.arange(d // 2, device=DEV) * (1 if c["layout"] == "half" else 2)
    second = first + (d // 2 if c["layout"] == "half" else 1)
    for i, (row, p0) in enumerate(zip(s["table"].tolist(), s["pos"].tolist())):
        par = s["parents"][i].tolist()
        places = [p0 + t if T > 200 else -1 if par[t] < -1 else p0 + len(_above(par, t)) - 1 for t in range(T)]
        places = torch.tensor(places, dtype=torch.float64, device=DEV)
        turn = torch.polar(torch.ones((), dtype=torch.float64, device=DEV), places[:, None] * rates)[None, :, None, :]
        x = s["qkv"][:, i].double()                           # [L, T, heads, hd]
        if c["norm"]:
            for lo, hi, gain in ((0, hq, s["q_gain"]), (hq, hq + hkv, s["k_gain"])):
                y = x[:, :, lo:hi]
                x[:, :, lo:hi] = y / torch.sqrt((y * y).sum(-1, keepdim=True) / hd + EPS) * gain.double()
        z = torch.complex(x[:, :, :hq + hkv, first], x[:, :, :hq + hkv, second]) * turn
        x[:, :, :hq + hkv, first], x[:, :, :hq + hkv, second] = z.real, z.imag
        x[:, places < 0] = 0.0
        out[:, i] = x[:, :, :hq]
        slot = p0 + torch.arange(T, device=DEV)
        page, r = torch.tensor(row, device=DEV)[slot // PAGE], slot % PAGE
        for which, at, lo in ((0, k_at, hq), (1, v_at, hq + hkv)):
            for l in range(c["layers"]):
                for h in range(hkv):
                    pool[page[:, None], l, which, h, at[r]] = x[l, :, lo + h]
    return {"q": out, "pool": pool}


def _exact_tree(s):
    c = s["c"]
    hq, hkv, hd = HEADS[c["heads"]]
    T, grp = c["nodes"], hq // hkv
    k_at, v_at = _tile_at(hd)
    out = torch.zeros(s["out"].shape, dtype=torch.float64, device=DEV)
    for i, (row, p0) in enumerate(zip(s["table"].tolist(), s["pos"].tolist())):
        par = s["parents"][i].tolist()
        see = torch.zeros((T, p0 + T), dtype=torch.bool)
        for t in range(T):
            if par[t] >= -1:
                see[t, :p0] = True
                see[t, [p0 + u for u in _above(par, t)]] = True
        live = torch.tensor([p >= -1 for p in par], device=DEV)
        see = see.to(DEV)[live]
        pages = torch.tensor(row[:_up(p0 + T)], device=DEV)
        for l in range(c["layers"]):
            for h in range(hkv):
                k, v = (s["pool"][pages, l, w, h].view(s["dt"])[:, a].double().reshape(-1, hd)[:p0 + T] for w, a in ((0, k_at), (1, v_at)))
                q = s["q"][l, i, live, h * grp:(h + 1) * grp].double().transpose(0, 1)
                x = torch.matmul(q, k.T) / math.sqrt(hd)
                w = torch.softmax(x.masked_fill(~see, -math.inf), -1)
                out[l, i, live, h * grp:(h + 1) * grp] = torch.matmul(w, v).transpose(0, 1)
    return {"out": out, "places": None}


def _exact_choose(s):
    c = s["c"]
    T, vocab = c["nodes"], c["vocab"]
    out, token = [], []
    for i, told in enumerate(s["history_len"].tolist()):
        text = s["history"][i, :told].long()
        par, tok = (None, None) if T == 1 else (s["parents"][i].tolist(), s["drafted"][i])
        for t in range(T):
            up = [] if T == 1 or par[t] < -1 else _above(par, t)
            mine = torch.cat([text, tok[up].long()]) if up else text
            n = torch.bincount(mine, minlength=vocab).double()
            x = s["logits"][i * T + t].double()
            x = torch.where(n > 0, torch.where(x > 0, x / c["repetition"], x * c["repetition"]) - c["presence"], x) - c["frequency"] * n
            if s["bias"] is not None:
                x = x + s["bias"].double()
            if s["allowed"] is not None:
                at = torch.arange(vocab, device=DEV)
                x[(s["allowed"][i * T + t, at // 32].long() >> (at % 32) & 1) == 0] = -math.inf
            out.append(x)
    return {"logits": torch.stack(out), "token": None}


def exact(case, seed):
    c = case
    if c["kind"] == "choose":
        return None if c["entries"] * c["nodes"] > 8000 else _exact_choose(_inputs(c, seed))
    n, hkv = len(_entries(c)), HEADS[c["heads"]][1]
    if n * hkv * c["layers"] > 20000:
        return None                                            # (minutes)
    s = _inputs(c, seed)
    if c["kind"] == "append":
        return _exact_append(s)
    if c["kind"] == "tree":
        return _exact_tree(s)
    # values are moved, none is computed
    i32 = dict(dtype=torch.int32, device=DEV)
    T, table, refs, length = c["nodes"], s["table"].tolist(), s["refs"].tolist(), s["len"].tolist()
    paths, counts, tokens = [], [], []
    k_at, v_at = _tile_at(HEADS[c["heads"]][2])
    for i, p0 in enumerate(s["pos"].tolist()):
        par, tok, ch = (s[k][i].tolist() for k in ("parents", "drafted", "chosen"))
        path = [0]
        while True:
            more = [t for t in range(1, T) if par[t] == path[-1] and tok[t] == ch[path[-1]]]
            if not more:
                break
            path.append(more[0])
        for k, t in enumerate(path):
            (pa, ra), (pb, rb) = (divmod(p0 + x, PAGE) for x in (t, k))
            for w, at in ((0, k_at), (1, v_at)):
                s["pool"][table[i][pb], :, w][..., at[rb]] = s["pool"][table[i][pa], :, w][..., at[ra]]
        for j in range(_up(p0 + len(path)), _up(length[i])):
            refs[table[i][j]] -= 1
            table[i][j] = -1
        length[i] = p0 + len(path)
        paths.append(path + [-1] * (T - len(path)))
        counts.append(len(path))
        tokens.append(ch[path[-1]])
    return {"path": torch.tensor(paths, **i32), "count": torch.tensor(counts, **i32), "token": torch.tensor(tokens, **i32),
            "pool": s["pool"], "table": torch.tensor(table, **i32), "refs": torch.tensor(refs, **i32),
            "len": torch.tensor(length, **i32)}
