"""The operators on a paged KV cache that several candidate action sequences of one observation
share, as cases that can be timed and checked: forking sequences, making room and appending new
tokens, attention that reads a shared prefix once for all, compacting the pool.

A page holds K and V of 32 positions for all layers, [layer][K, V][kv head][32 * head_dim], a
head's 32 positions in the order in which the matrix cores take them:
  K  [head_dim / 16][2][32 positions][8]          feature 16 a + 8 g + e of position r at [a][g][r][e]
  V  [head_dim / 32][2][2][32 features][2][4]     feature 32 b + f of position 16 t + 8 i + 4 g + e at [b][t][g][f][i][e]
table [sequences, pages per sequence] names a sequence's pages (-1 behind its last), len its
positions, refs how many table entries name a page.

`run` is one pass as a program makes it, in elementary torch operations or (own) by the library.
Sizes of sequences are functions of the case, values come from the seed.  Positions that no
token was ever written to hold NaN patterns, as fresh memory may."""
import math

import torch

own = False

DEV = "cuda:0"
PAGE = 32
# query heads, kv heads, head_dim: the decoder shapes of this repository, and two generic layouts
HEADS = {"tiny": (4, 4, 64), "7b": (32, 32, 128), "gqa": (12, 2, 128), "g4": (16, 4, 64), "mqa": (8, 1, 128)}
DTYPE = {"bf16": torch.bfloat16, "f16": torch.float16}


def listed():
    return [
        # one token of two candidates of the smoke shape: launches and latency
        dict(name="attend_tiny", kind="attend", heads="tiny", dtype="f16", layers=2, groups=1, cands=2, prefix=80,
             suffix=3, tokens=1),
        # a decode step of 3 to 8 candidates for each of 32 environments, grouped queries
        dict(name="attend_gqa_32", kind="attend", heads="gqa", dtype="bf16", layers=4, groups=32, cands=8, prefix=304,
             suffix=6, tokens=1),
        # 16 candidate chunks of 56 action rows over one two-view observation
        dict(name="attend_chunk", kind="attend", heads="7b", dtype="f16", layers=2, groups=1, cands=16, prefix=1057,
             suffix=1, tokens=56),
        # a long history that 48 candidates share, odd length
        dict(name="attend_long", kind="attend", heads="7b", dtype="f16", layers=2, groups=1, cands=48, prefix=32801,
             suffix=37, tokens=1),
        # K/V of one decoded token of 8 candidates, and of a chunk of 56 rows of 32 candidates
        dict(name="append_7b_8", kind="append", heads="7b", dtype="f16", layers=4, groups=2, cands=4, prefix=288,
             suffix=6, tokens=1),
        dict(name="append_gqa_chunk", kind="append", heads="gqa", dtype="bf16", layers=4, groups=8, cands=4, prefix=304,
             suffix=1, tokens=56),
        # candidates of a step: the full pages shared, the last one copied; and two whole copies
        # (a stream whose positions will be rewritten in place)
        dict(name="fork_7b", kind="fork", heads="7b", dtype="f16", layers=32, groups=2, cands=8, prefix=303,
             suffix=0, tokens=1, deep=False),
        dict(name="fork_deep_gqa", kind="fork", heads="gqa", dtype="bf16", layers=28, groups=8, cands=2, prefix=304,
             suffix=0, tokens=1, deep=True),
        # a pool after many steps, half and a tenth of it live
        dict(name="compact_7b_half", kind="compact", heads="7b", dtype="f16", layers=8, pages=301, live=0.5),
        dict(name="compact_gqa_sparse", kind="compact", heads="gqa", dtype="bf16", layers=4, pages=5003, live=0.1),
        # all of it together: fork, room for new tokens, append and attention per layer, free
        dict(name="turn_tiny", kind="turn", heads="tiny", dtype="f16", layers=2, groups=1, cands=4, prefix=80,
             suffix=0, tokens=1, deep=False),
        dict(name="turn_7b", kind="turn", heads="7b", dtype="f16", layers=4, groups=2, cands=8, prefix=601,
             suffix=0, tokens=8, deep=False),
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
        kind = rng.choice(["attend", "attend", "attend", "append", "fork", "compact", "turn"])
        c = dict(kind=kind, heads=rng.choice(["tiny", "7b", "7b", "gqa", "gqa", "g4", "mqa"]), dtype=rng.choice(["f16", "bf16"]))
        if kind == "compact":
            c.update(layers=rng.randint(1, 8), pages=log_int(40, 6000), live=round(rng.uniform(0.05, 0.95), 2))
        else:
            c.update(layers=rng.randint(1, 4), groups=log_int(1, 32), cands=log_int(1, 64),
                     prefix=log_int(1, 33000 if kind == "attend" else 1100), suffix=rng.randint(0, 70), tokens=1)
            if rng.random() < 0.4:
                c["tokens"] = log_int(2, 60)
            if kind in ("fork", "turn"):
                c.update(suffix=0, deep=rng.random() < 0.3)
            if kind == "fork":
                c.update(layers=rng.randint(1, 32), tokens=1)
        w = work(c)
        if w["flops"] <= top["flops"] and w["bytes"] <= top["bytes"] and _pool_bytes(c) <= 6e9 and _plain_bytes(c) <= 12e9:
            return c


# ------------------------------------------------------------------------------------------
# sizes, from the case alone
# ------------------------------------------------------------------------------------------
def _prefixes(c):
    """Positions of every group's common prefix: the first has the longest."""
    return [max(1, c["prefix"] - 11 * g % 37 - (g % 5 == 4) * (c["prefix"] // 3)) for g in range(c["groups"])]


def _members(c):
    """Candidates of every group."""
    return [max(1, c["cands"] - g * 3 % (c["cands"] // 2 + 1)) for g in range(c["groups"])]


def _entries(c):
    """(group, prefix, tokens of its own before the new ones) of every candidate, group by group."""
    out = []
    for g, (p, m) in enumerate(zip(_prefixes(c), _members(c))):
        for k in range(m):
            out.append((g, p, (c["suffix"] + 5 * k) % (c["suffix"] + 1)))
    return out


def _page_elems(c):
    _, hkv, hd = HEADS[c["heads"]]
    return c["layers"] * 2 * hkv * PAGE * hd


def _up(x):
    return -(-x // PAGE)


def _page_counts(c):
    """-> pages in the pool, pages per sequence, sequences."""
    if c["kind"] == "compact":
        return c["pages"], 16, max(1, int(c["pages"] * c["live"]) // 8)
    ent, most = _entries(c), c["prefix"] + c["suffix"] + c["tokens"]
    shared = sum(_up(p) for p in _prefixes(c))
    each = [_up(p + s + c["tokens"]) - (0 if c.get("deep") else p // PAGE) for _, p, s in ent]
    return shared + sum(each) + 7, _up(most) + 1, c["groups"] + len(ent) + 3


def _pool_bytes(c):
    return _page_counts(c)[0] * _page_elems(c) * 2


def _plain_bytes(c):
    """Largest 32-bit score array of the plain form."""
    if c["kind"] not in ("attend", "turn"):
        return 0
    ent = _entries(c)
    return 4 * c["groups"] * max(_members(c)) * c["tokens"] * HEADS[c["heads"]][0] * c["prefix"]


def _live_split(c):
    """compact: pages that are live, of the pool's first, in an order that the seed shuffles."""
    return max(1, int(c["pages"] * c["live"]))


def work(case):
    c = case
    hq, hkv, hd = HEADS[c["heads"]]
    page = _page_elems(c) * 2
    if c["kind"] == "compact":
        n, seqs = c["pages"], _page_counts(c)[2]
        live = _live_split(c) - 5 * (seqs // 3)              # (a third of the sequences share five pages)
        return {"bytes": int(2 * page * live * (n - live) / n) + 8 * n, "flops": 0}
    ent, T, L = _entries(c), c["tokens"], c["layers"]
    row = hkv * hd * 2 * 2                                   # K and V of one position and layer
    out = {"bytes": 0, "flops": 0}
    if c["kind"] in ("fork", "turn"):
        pages = sum(_up(p) for _, p, _ in ent) if c["deep"] else sum(p % PAGE != 0 for _, p, _ in ent)
        read = sum(_up(p) for p in _prefixes(c)) if c["deep"] else sum(p % PAGE != 0 for p in _prefixes(c))
        out["bytes"] += (pages + read) * page
    if c["kind"] in ("append", "turn"):
        out["bytes"] += 2 * L * len(ent) * T * row
    if c["kind"] in ("attend", "turn"):
        shared = sum(p // PAGE * PAGE for p in _prefixes(c))
        private = sum(p % PAGE + s + T for _, p, s in ent)
        if c.get("deep"):                                    # nothing is shared between whole copies
            shared, private = 0, sum(p + s + T for _, p, s in ent)
        seen = sum(T * (p + s) + T * (T + 1) // 2 for _, p, s in ent)
        out["bytes"] += L * ((shared + private) * row + 2 * len(ent) * T * hq * hd * 2)
        out["flops"] += L * 4 * hd * hq * seen
    return out


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


def _k_tiles(x):
    """[..., 32, hd] -> [..., 32 * hd] in the order of a K tile."""
    *lead, _, hd = x.shape
    return x.reshape(*lead, PAGE, hd // 16, 2, 8).movedim(-4, -2).reshape(*lead, PAGE * hd)


def _v_tiles(x):
    *lead, _, hd = x.shape
    y = x.reshape(*lead, 2, 2, 2, 4, hd // 32, 32)           # t, i, g, e, b, f
    n = len(lead)
    return y.permute(*range(n), n + 4, n, n + 2, n + 5, n + 1, n + 3).reshape(*lead, PAGE * hd)


def _inputs(c, seed):
    """Everything that a program has in hand, as plain tensors."""
    hq, hkv, hd = HEADS[c["heads"]]
    dt, T, L = DTYPE[c["dtype"]], c.get("tokens", 1), c["layers"]
    n_pages, max_pages, max_seqs = _page_counts(c)
    s = {"c": c, "dt": dt}
    i32 = dict(dtype=torch.int32, device=DEV)
    pool = torch.full((n_pages, L, 2, hkv, PAGE * hd), -1, dtype=torch.int16, device=DEV)   # NaN patterns
    order = torch.randperm(n_pages, generator=_gen(seed, 1), device=DEV).tolist()           # where a long run left them
    table, refs, length = [[-1] * max_pages for _ in range(max_seqs)], [0] * n_pages, [0] * max_seqs
    if c["kind"] == "compact":
        live = order[:_live_split(c)]
        at = 0
        for q in range(max_seqs):                             # eight pages each, the last one the rest
            mine = live[at:at + 8] if q + 1 < max_seqs else live[at:at + 16]
            at += len(mine)
            if q % 3 == 2:                                    # every third shares the first pages of the one before
                mine = table[q - 1][:5] + mine[5:]
            table[q][:len(mine)] = mine
            length[q] = PAGE * len(mine) - (7 * q % PAGE if mine else 0)
        for row in table:
            for p in row:
                if p >= 0:
                    refs[p] += 1
        pool[torch.tensor(live, device=DEV)] = torch.randn((len(live), L, 2, hkv, PAGE * hd), generator=_gen(seed, 2),
                                                           device=DEV, dtype=dt).view(torch.int16)
        s["live"] = torch.zeros(1, **i32)
    else:
        ent, G = _entries(c), c["groups"]
        free = iter(order)
        fresh = []                                            # (page, positions written)

        def take(filled):
            p = next(free)
            fresh.append((p, filled))
            return p

        # sources: sequences 0 .. G - 1; candidates behind them
        for g, p in enumerate(_prefixes(c)):
            length[g] = p
            for j in range(_up(p)):
                table[g][j] = take(min(PAGE, p - j * PAGE))
        if c["kind"] in ("attend", "append"):
            for i, (g, p, suf) in enumerate(ent):
                q, held = G + i, p + suf + T
                done = held if c["kind"] == "attend" else p + suf
                length[q] = held
                for j in range(_up(held)):
                    shared = j < p // PAGE
                    table[q][j] = table[g][j] if shared else take(min(PAGE, max(0, done - j * PAGE)))
        for row in table:
            for p in row:
                if p >= 0:
                    refs[p] += 1
        pages = torch.tensor([p for p, _ in fresh], device=DEV)
        filled = torch.tensor([f for _, f in fresh], device=DEV)
        g2 = _gen(seed, 2)
        step = max(1, int(2e8) // (2 * hkv * PAGE * hd))      # (in pieces: the 32-bit draws are large)
        for l in range(L):
            for a in range(0, len(fresh), step):
                x = torch.randn((len(pages[a:a + step]), 2, hkv, PAGE, hd), generator=g2, device=DEV).to(dt)
                hole = torch.arange(PAGE, device=DEV)[None, :] >= filled[a:a + step, None]
                x = x.view(torch.int16).masked_fill_(hole[:, None, None, :, None], -1)
                pool[pages[a:a + step], l] = torch.stack([_k_tiles(x[:, 0]), _v_tiles(x[:, 1])], 1)
        s["src"] = torch.tensor([g for g, _, _ in ent], **i32)
        s["seqs"] = torch.arange(G, G + len(ent), **i32)
        s["pos"] = torch.tensor([p + suf for _, p, suf in ent], **i32)
        n = len(ent)
        # sharp enough that a few dozen positions carry most of the weight
        s["q"] = (2.5 * torch.randn((L, n, T, hq, hd), generator=_gen(seed, 3), device=DEV)).to(dt)
        s["k"] = torch.randn((L, n, T, hkv, hd), generator=_gen(seed, 4), device=DEV).to(dt)
        s["v"] = torch.randn((L, n, T, hkv, hd), generator=_gen(seed, 5), device=DEV).to(dt)
        s["out"] = torch.zeros((L, n, T, hq, hd), dtype=dt, device=DEV)
    s["pool"] = pool
    s["table"], s["refs"], s["len"] = torch.tensor(table, **i32), torch.tensor(refs, **i32), torch.tensor(length, **i32)
    if c["kind"] == "compact":
        s["table0"], s["refs0"] = s["table"].clone(), s["refs"].clone()
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    if own:
        import paper_2502_02175_amd as V
        c = case
        hq, hkv, hd = HEADS[c["heads"]]
        s["V"] = V
        s["pages"] = V.pages(c["layers"], hkv, hd, V.OPERAND_F16 if c["dtype"] == "f16" else V.OPERAND_BF16,
                             s["pool"], s["refs"], s["table"], s["len"])
        if c["kind"] in ("attend", "turn"):
            n = s["seqs"].numel()
            s["ws"] = torch.empty(V.vlac_attend_workspace_bytes(s["pages"], n, c["tokens"], hq), dtype=torch.uint8, device=DEV)
        if c["kind"] == "turn":
            s["pos"] = torch.empty_like(s["pos"])
    return s


# ------------------------------------------------------------------------------------------
# one pass
# ------------------------------------------------------------------------------------------
def run(state):
    s, c = state, state["c"]
    kind = c["kind"]
    if kind == "compact":
        s["refs"].copy_(s["refs0"])                           # (the pool as it was before the last pass)
        s["table"].copy_(s["table0"])
        (_own_compact if own else _compact)(s)
        return {"pool": s["pool"], "refs": s["refs"], "table": s["table"], "live": s["live"]}
    if kind == "fork":
        (_own_fork if own else _fork)(s)
        return {"pool": s["pool"], "refs": s["refs"], "table": s["table"], "len": s["len"]}
    if kind == "append":
        (_own_append if own else _append)(s)
        return {"pool": s["pool"]}
    if kind == "attend":
        (_own_attend if own else _attend)(s)
        return {"out": s["out"]}
    (_own_turn if own else _turn)(s)
    return {"out": s["out"], "pos": s["pos"], "pool": s["pool"], "refs": s["refs"], "table": s["table"], "len": s["len"]}


def _own_compact(s):
    s["V"].vlac_pages_compact(s["pages"], s["live"])


def _own_fork(s):
    s["V"].vlac_pages_fork(s["pages"], s["src"], s["seqs"], s["seqs"].numel(), s["c"]["deep"])


def _own_append(s):
    n, T = s["seqs"].numel(), s["c"]["tokens"]
    for l in range(s["c"]["layers"]):
        s["V"].vlac_pages_append(s["pages"], l, s["seqs"], s["pos"], n, T, s["k"][l], s["v"][l])


def _own_attend(s):
    V, n, T, hq = s["V"], s["seqs"].numel(), s["c"]["tokens"], HEADS[s["c"]["heads"]][0]
    V.vlac_attend_plan(s["pages"], s["seqs"], s["pos"], n, T, hq, s["src"], s["ws"])
    for l in range(s["c"]["layers"]):
        V.vlac_attend_shared(s["pages"], l, n, T, hq, s["q"][l], s["out"][l], s["ws"])


def _own_turn(s):
    V, n, T, hq = s["V"], s["seqs"].numel(), s["c"]["tokens"], HEADS[s["c"]["heads"]][0]
    _own_fork(s)
    V.vlac_pages_extend(s["pages"], s["seqs"], n, T, s["pos"])
    V.vlac_attend_plan(s["pages"], s["seqs"], s["pos"], n, T, hq, s["src"], s["ws"])
    for l in range(s["c"]["layers"]):
        V.vlac_pages_append(s["pages"], l, s["seqs"], s["pos"], n, T, s["k"][l], s["v"][l])
        V.vlac_attend_shared(s["pages"], l, n, T, hq, s["q"][l], s["out"][l], s["ws"])
    V.vlac_pages_free(s["pages"], s["seqs"], n)


# the plain forms ---------------------------------------------------------------------------
def _count(s, rows, mask, by):
    """refs of the named pages += by."""
    s["refs"].index_add_(0, rows.clamp(min=0).reshape(-1), (mask.to(torch.int32) * by).reshape(-1))


def _free_pages(s):
    """Page indices, the free ones first, ascending."""
    return torch.sort((s["refs"] != 0).to(torch.int8), stable=True).indices.to(torch.int32)


def _release(s, seqs):
    rows = s["table"][seqs]
    _count(s, rows, rows >= 0, -1)
    s["table"][seqs] = -1
    s["len"][seqs] = 0


def _fork(s):
    src, dst = s["src"].long(), s["seqs"].long()
    _release(s, dst)
    ln, rows = s["len"][src], s["table"][src]
    col = torch.arange(rows.shape[1], device=DEV)[None, :]
    count = ((ln + PAGE - 1) // PAGE)[:, None]
    if s["c"]["deep"]:
        fresh = col < count
    else:
        fresh = (col == count - 1) & (ln % PAGE != 0)[:, None]
    kept = (col < count) & ~fresh
    rank = (fresh.reshape(-1).cumsum(0) - 1).clamp(min=0).reshape(fresh.shape)
    pages = _free_pages(s)[rank]
    new = torch.where(fresh, pages, torch.where(kept, rows, -1))
    _count(s, new, new >= 0, 1)
    s["table"][dst] = new
    s["len"][dst] = ln
    s["pool"][pages[fresh].long()] = s["pool"][rows[fresh].long()]


def _extend(s, tokens):
    seqs = s["seqs"].long()
    pos, rows = s["len"][seqs], s["table"][seqs]
    col = torch.arange(rows.shape[1], device=DEV)[None, :]
    fresh = (col >= ((pos + PAGE - 1) // PAGE)[:, None]) & (col < ((pos + tokens + PAGE - 1) // PAGE)[:, None])
    rank = (fresh.reshape(-1).cumsum(0) - 1).clamp(min=0).reshape(fresh.shape)
    pages = _free_pages(s)[rank]
    _count(s, pages, fresh, 1)
    s["table"][seqs] = torch.where(fresh, pages, rows)
    s["len"][seqs] = pos + tokens
    s["pos"].copy_(pos)


def _append(s, layers=None):
    _, hkv, hd = HEADS[s["c"]["heads"]]
    T = s["c"]["tokens"]
    at = (s["pos"].long()[:, None] + torch.arange(T, device=DEV)[None, :])
    page = s["table"].long()[s["seqs"].long()[:, None], at // PAGE].reshape(-1)
    r = (at % PAGE).reshape(-1)
    pool = s["pool"]
    for l in range(s["c"]["layers"]) if layers is None else layers:
        kv = pool[:, l, 0].view(-1, hkv, hd // 16, 2, PAGE, 8)
        kv[page, :, :, :, r] = s["k"][l].view(torch.int16).reshape(-1, hkv, hd // 16, 2, 8)
        vv = pool[:, l, 1].view(-1, hkv, hd // 32, 2, 2, 32, 2, 4)
        vv[page, :, :, r // 16, r // 4 % 2, :, r // 8 % 2, r % 4] = s["v"][l].view(torch.int16).reshape(-1, hkv, hd // 32, 32)


def _gather(s, layer, which, pages):
    """[...] page indices -> K or V rows in 32 bits, [..., 32, hkv, hd]."""
    _, hkv, hd = HEADS[s["c"]["heads"]]
    x = s["pool"][pages, layer, which].view(s["dt"]).float()
    lead = x.shape[:-2]
    n = len(lead)
    if which == 0:
        y = x.view(*lead, hkv, hd // 16, 2, PAGE, 8).permute(*range(n), n + 3, n, n + 1, n + 2, n + 4)
    else:
        y = x.view(*lead, hkv, hd // 32, 2, 2, 32, 2, 4).permute(*range(n), n + 2, n + 5, n + 3, n + 6, n, n + 1, n + 4)
    return y.reshape(*lead, PAGE, hkv, hd)


def _attend(s, layers=None):
    """The common pages of a group once for all its candidates, the rest of each for itself."""
    c = s["c"]
    hq, hkv, hd = HEADS[c["heads"]]
    T, G, M, grp = c["tokens"], c["groups"], max(_members(c)), hq // hkv
    members, ent = _members(c), _entries(c)
    if "slots" not in s:                                      # where an entry stands in [group, candidate]: plan, kept
        first = [sum(members[:g]) for g in range(G)]
        s["slots"] = torch.tensor([g * M + i - first[g] for i, (g, _, _) in enumerate(ent)], device=DEV)
        common = [0 if c.get("deep") else p // PAGE for p in _prefixes(c)]
        s["common"] = torch.tensor(common, device=DEV)
        s["leaders"] = torch.tensor(first, device=DEV)
        s["own_from"] = torch.tensor([common[g] for g, _, _ in ent], device=DEV)
        s["n_common"] = max(common)
        s["n_own"] = max(_up(p + suf + T) - common[g] for g, p, suf in ent)
    seqs, pos, table = s["seqs"].long(), s["pos"].long(), s["table"].long()
    n = seqs.numel()
    own_col = s["own_from"][:, None] + torch.arange(s["n_own"], device=DEV)[None, :]
    own_pages = table[seqs[:, None], own_col.clamp(max=table.shape[1] - 1)].clamp(min=0)
    own_at = (own_col[:, :, None] * PAGE + torch.arange(PAGE, device=DEV)).reshape(n, -1)
    last = pos[:, None] + torch.arange(T, device=DEV)[None, :]
    own_seen = own_at[:, None, :] <= last[:, :, None]          # [n, T, own]
    written = own_at < (pos + T)[:, None]
    pre_pages = table[seqs[s["leaders"]]][:, :s["n_common"]].clamp(min=0)
    pre_seen = torch.arange(s["n_common"] * PAGE, device=DEV)[None, :] < (s["common"] * PAGE)[:, None]
    scale = 1.0 / math.sqrt(hd)
    for l in range(c["layers"]) if layers is None else layers:
        q = s["q"][l].float()                                  # [n, T, hq, hd]
        qh = q.view(n, T, hkv, grp, hd).permute(0, 2, 1, 3, 4)  # [n, hkv, T, grp, hd]
        ko, vo = (_gather(s, l, w, own_pages).reshape(n, -1, hkv, hd) for w in (0, 1))
        vo = torch.where(written[:, :, None, None], vo, 0.0)
        so = torch.matmul(qh.reshape(n, hkv, T * grp, hd), ko.permute(0, 2, 3, 1).contiguous()) * scale
        so = torch.where(own_seen[:, None, :, None, :], so.view(n, hkv, T, grp, -1), -math.inf)
        m = so.amax(-1)
        if s["n_common"]:
            kp, vp = (_gather(s, l, w, pre_pages).reshape(G, -1, hkv, hd) for w in (0, 1))
            vp = torch.where(pre_seen[:, :, None, None], vp, 0.0)
            qg = q.new_zeros((G * M, hkv, T, grp, hd))
            qg[s["slots"]] = qh
            qg = qg.view(G, M, hkv, T * grp, hd).permute(0, 2, 1, 3, 4).reshape(G, hkv, M * T * grp, hd)
            sp = torch.matmul(qg, kp.permute(0, 2, 3, 1).contiguous()) * scale
            sp = torch.where(pre_seen[:, None, None, :], sp, -math.inf)
            mp = sp.amax(-1)

            def per_entry(x):                                  # [G, hkv, M * T * grp, ...] -> [n, hkv, T, grp, ...]
                x = x.view(G, hkv, M, T, grp, -1).permute(0, 2, 1, 3, 4, 5)
                return x.reshape(G * M, hkv, T, grp, -1)[s["slots"]]

            top = torch.maximum(m, per_entry(mp)[..., 0])
            tg = q.new_zeros((G * M, hkv, T, grp))
            tg[s["slots"]] = top
            tg = tg.view(G, M, hkv, T * grp).permute(0, 2, 1, 3).reshape(G, hkv, M * T * grp)
            pp = torch.exp(sp - tg[..., None])
            num = per_entry(torch.matmul(pp, vp.permute(0, 2, 1, 3).contiguous()))
            den = per_entry(pp.sum(-1))[..., 0]
            m = top
        else:
            num = den = 0.0
        po = torch.exp(so - m[..., None])
        num = num + torch.matmul(po.view(n, hkv, T * grp, -1), vo.permute(0, 2, 1, 3).contiguous()).view(n, hkv, T, grp, hd)
        den = den + po.sum(-1)
        s["out"][l] = (num / den[..., None]).permute(0, 2, 1, 3, 4).reshape(n, T, hq, hd).to(s["dt"])


def _compact(s):
    refs = s["refs"]
    n = refs.numel()
    held = refs > 0
    live = held.sum()
    at = torch.arange(n, device=DEV)
    src = torch.nonzero(held & (at >= live)).reshape(-1)
    dst = torch.nonzero(~held & (at < live)).reshape(-1)
    s["pool"][dst] = s["pool"][src]
    refs[dst] = refs[src]
    refs[src] = 0
    to = at.to(torch.int32)
    to[src] = dst.to(torch.int32)
    s["table"].copy_(torch.where(s["table"] >= 0, to[s["table"].clamp(min=0).long()], -1))
    s["live"][0] = live


def _turn(s):
    _fork(s)
    _extend(s, s["c"]["tokens"])
    for l in range(s["c"]["layers"]):
        _append(s, [l])
        _attend(s, [l])
    _release(s, s["seqs"].long())


# ------------------------------------------------------------------------------------------
# the definition, in 64 bits and one sequence (or one group) at a time
# ------------------------------------------------------------------------------------------
class _Book:
    """Tables and reference counts as Python lists."""

    def __init__(self, s):
        self.table, self.refs, self.len = s["table"].tolist(), s["refs"].tolist(), s["len"].tolist()

    def lowest(self):
        p = self.refs.index(0)
        self.refs[p] = 1
        return p

    def drop(self, q):
        for j, p in enumerate(self.table[q]):
            if p >= 0:
                self.refs[p] -= 1
            self.table[q][j] = -1
        self.len[q] = 0

    def out(self):
        i32 = dict(dtype=torch.int32, device=DEV)
        return torch.tensor(self.refs, **i32), torch.tensor(self.table, **i32), torch.tensor(self.len, **i32)


def _exact_fork(s, book):
    src, dst = s["src"].tolist(), s["seqs"].tolist()
    for q in dst:
        book.drop(q)
    for a, b in zip(src, dst):
        n = book.len[a]
        for j in range(_up(n)):
            p = book.table[a][j]
            if s["c"]["deep"] or (j + 1) * PAGE > n:
                f = book.lowest()
                s["pool"][f] = s["pool"][p]
                p = f
            else:
                book.refs[p] += 1
            book.table[b][j] = p
        book.len[b] = n


def _exact_append(s, table):
    _, hkv, hd = HEADS[s["c"]["heads"]]
    T, pool = s["c"]["tokens"], s["pool"]
    f = torch.arange(hd, device=DEV)
    bits = lambda x: x.view(torch.int16)
    for i, (q, p0) in enumerate(zip(s["seqs"].tolist(), s["pos"].tolist())):
        for t in range(T):
            page, r = table[q][(p0 + t) // PAGE], (p0 + t) % PAGE
            k_at = f // 16 * 512 + f // 8 % 2 * 256 + r * 8 + f % 8
            v_at = f // 32 * 1024 + r // 16 * 512 + r // 4 % 2 * 256 + f % 32 * 8 + r // 8 % 2 * 4 + r % 4
            pool[page, :, 0, :, k_at] = bits(s["k"][:, i, t])
            pool[page, :, 1, :, v_at] = bits(s["v"][:, i, t])


def _exact_attend(s, table):
    c = s["c"]
    hq, hkv, hd = HEADS[c["heads"]]
    T, grp, dt = c["tokens"], hq // hkv, s["dt"]
    f = torch.arange(hd, device=DEV)
    r = torch.arange(PAGE, device=DEV)[:, None]
    k_at = (f // 16 * 512 + f // 8 % 2 * 256 + f % 8)[None, :] + r * 8
    v_at = (f // 32 * 1024 + f % 32 * 8)[None, :] + r // 16 * 512 + r // 4 % 2 * 256 + r // 8 % 2 * 4 + r % 4
    out = torch.zeros(s["out"].shape, dtype=torch.float64, device=DEV)
    seqs, pos, groups = s["seqs"].tolist(), s["pos"].tolist(), s["src"].tolist()
    lo = 0
    while lo < len(seqs):
        hi = lo
        while hi < len(seqs) and groups[hi] == groups[lo]:
            hi += 1
        rows = [table[seqs[i]][:_up(pos[i] + T)] for i in range(lo, hi)]
        common = 0
        while all(common < pos[lo + x] // PAGE and row[common] == rows[0][common] for x, row in enumerate(rows)):
            common += 1
        for l in range(c["layers"]):
            for h in range(hkv):
                def rows_of(pages, which):
                    x = s["pool"][torch.tensor(pages, device=DEV), l, which, h].view(dt)
                    return x[:, k_at if which == 0 else v_at].double().reshape(-1, hd)

                q = s["q"][l, lo:hi, :, h * grp:(h + 1) * grp].double() / math.sqrt(hd)
                if common:
                    kp, vp = rows_of(rows[0][:common], 0), rows_of(rows[0][:common], 1)
                    sp = q.reshape(-1, hd) @ kp.T
                    sp = sp.view(hi - lo, T * grp, -1)
                for x, i in enumerate(range(lo, hi)):
                    own_pages = rows[x][common:]
                    ko, vo = rows_of(own_pages, 0), rows_of(own_pages, 1)
                    kept = pos[i] + T - common * PAGE
                    so = (q[x].reshape(-1, hd) @ ko[:kept].T).view(T, grp, kept)
                    at = common * PAGE + torch.arange(kept, device=DEV)
                    so = so.masked_fill(at[None, None, :] > pos[i] + torch.arange(T, device=DEV)[:, None, None], -math.inf)
                    so = so.view(T * grp, kept)
                    both = torch.cat([sp[x], so], 1) if common else so
                    w = torch.softmax(both, 1)
                    y = w[:, common * PAGE:] @ vo[:kept]
                    if common:
                        y = y + w[:, :common * PAGE] @ vp
                    out[l, i, :, h * grp:(h + 1) * grp] = y.view(T, grp, hd)
        lo = hi
    return out


def exact(case, seed):
    c = case
    if c["kind"] in ("attend", "turn") and c["layers"] * HEADS[c["heads"]][1] * len(_entries(c)) > 20000:
        return None                                            # (minutes)
    s = _inputs(c, seed)
    if c["kind"] == "attend":
        return {"out": _exact_attend(s, s["table"].tolist())}
    if c["kind"] == "append":
        _exact_append(s, s["table"].tolist())
        return {"pool": s["pool"]}
    book = _Book(s)
    if c["kind"] == "compact":
        live = sum(x > 0 for x in book.refs)
        holes = iter([p for p in range(live) if book.refs[p] == 0])
        to = {}
        for p in range(live, len(book.refs)):
            if book.refs[p] > 0:
                to[p] = next(holes)
                s["pool"][to[p]] = s["pool"][p]
                book.refs[to[p]], book.refs[p] = book.refs[p], 0
        book.table = [[to.get(p, p) for p in row] for row in book.table]
        refs, table, _ = book.out()
        return {"pool": s["pool"], "refs": refs, "table": table, "live": torch.tensor([live], dtype=torch.int32, device=DEV)}
    _exact_fork(s, book)
    if c["kind"] == "fork":
        refs, table, length = book.out()
        return {"pool": s["pool"], "refs": refs, "table": table, "len": length}
    seqs = s["seqs"].tolist()
    pos = [book.len[q] for q in seqs]
    for q in seqs:
        for j in range(_up(book.len[q]), _up(book.len[q] + c["tokens"])):
            book.table[q][j] = book.lowest()
        book.len[q] += c["tokens"]
    s["pos"] = torch.tensor(pos, dtype=torch.int32, device=DEV)
    _exact_append(s, book.table)
    out = _exact_attend(s, book.table)
    for q in seqs:
        book.drop(q)
    refs, table, length = book.out()
    return {"out": out, "pos": s["pos"], "pool": s["pool"], "refs": refs, "table": table, "len": length}
