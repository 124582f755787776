"""The operators on drafted tokens together, as a decoder uses them: room, plan, per layer append and attention, choice, accepted path, kept
pages, turn after turn, against the same decoder fed one token at a time; in a captured graph; on two streams."""
import math
import random

import pytest

import drafts_model as M
import paper_2502_02175_amd as V
from pages_model import OK, PAGE, k_tile_at, pages_of, v_tile_at

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
VOCAB = 40


def i32(x):
    import torch
    return torch.tensor(x, dtype=torch.int32, device=DEV)


class Toy:
    """A decoder whose layers' projections are tables over tokens, with a joint row [q, k, v]; its logits are what the layers'
    attention gives times a head, plus 8 for the token that always follows.  So attention moves the logits and decides
    nothing, and a choice is never near a border."""

    def __init__(self, hq, hkv, hd, operand, layers, seed, norm):
        import torch
        g = torch.Generator(device=DEV)
        g.manual_seed(seed)
        self.hq, self.hkv, self.hd, self.layers, self.operand = hq, hkv, hd, layers, operand
        self.dt = torch.bfloat16 if operand == 0 else torch.float16
        self.qkv = torch.randn((layers, VOCAB, hq + 2 * hkv, hd), generator=g, device=DEV).clamp(-3, 3).to(self.dt)
        self.head = torch.randn((layers, hq * hd, VOCAB), generator=g, device=DEV, dtype=torch.float64) / math.sqrt(layers * hq * hd)
        self.after = torch.randperm(VOCAB, generator=g, device=DEV)
        self.gains = [(1 + 0.2 * torch.randn(hd, generator=g, device=DEV)).bfloat16() for _ in "qk"] if norm else [None, None]
        self.rot = V.rotary(hd, V.ROTARY_HALF, 1e4, 4.0, 64, 1.0, 4.0)
        # The attention's result is off by half a step for the weights and one for itself (of at most 3, V's largest), and by its fp32
        # sums: hd products of a score whose sizes add up to 3 x 3 x sqrt(hd) at most (with norm 1.8 x 1.8), up to 200 weights.
        step, size = torch.finfo(self.dt).eps / 2, (3.3 if norm else 9) * math.sqrt(hd)
        fp32 = 2.0 ** -23 * (2 * (hd + 2) * size + 2 * 200 + 16)
        self.tol = (2 * step + fp32) * 3 * float(self.head.abs().sum(1).amax(1).sum()) + 16 * 2.0 ** -23
        # keys and queries: a step (rounding may part the two), and what fp32 makes of a norm, a rotation and values of up to 6
        self.step, self.kq = 2 * step, 12 * ((hd + 4) / 2 + 16) * 2.0 ** -24

    def logits(self, tokens, outs):
        """tokens [rows] -> fp32 [rows, VOCAB]."""
        import torch
        x = torch.zeros((tokens.numel(), VOCAB), dtype=torch.float64, device=DEV)
        for l in range(self.layers):
            x += outs[l].reshape(tokens.numel(), -1).double() @ self.head[l]
        x[torch.arange(tokens.numel(), device=DEV), self.after[tokens.long().reshape(-1)]] += 8.0
        return x.float()


class Drafts:
    """A batch of sequences of a pool whose trees are checked, with every buffer in one place (so that a turn can be captured)."""

    def __init__(self, toy, n, T, stem, turns, seed):
        import torch
        self.toy, self.n, self.T = toy, n, T
        rng = random.Random(seed)
        self.texts = [[rng.randrange(VOCAB) for _ in range(stem + 3 * i)] for i in range(n)]
        most = max(len(t) for t in self.texts) + turns * T
        self.p = V.new_pages(toy.layers, toy.hkv, toy.hd, toy.operand, n * pages_of(most) * 2 + 4, 2 * n, pages_of(most) + 1, DEV)
        self.p.tensors[0].fill_(0xFF)                           # NaN where nothing was written
        self.seqs = i32(range(n))
        self.pos, self.token, self.count = i32([0] * n), i32([0] * n), i32([0] * n)
        self.parents, self.drafted, self.places, self.path = (torch.zeros((n, T), dtype=torch.int32, device=DEV) for _ in range(4))
        self.chosen = torch.zeros(n * T, dtype=torch.int32, device=DEV)
        self.raw, self.ruled = (torch.zeros((n * T, VOCAB), device=DEV) for _ in range(2))
        self.outs, self.q = (torch.zeros((toy.layers, n, T, toy.hq, toy.hd), dtype=toy.dt, device=DEV) for _ in range(2))
        self.ws = torch.empty(V.vlac_attend_tree_workspace_bytes(self.p, n, T, toy.hq), dtype=torch.uint8, device=DEV)
        self.ws2 = torch.empty(V.vlac_choose_workspace_bytes(n * T, VOCAB), dtype=torch.uint8, device=DEV)
        self.history = torch.zeros((n, most), dtype=torch.int32, device=DEV)
        self.told = i32([0] * n)
        self.allowed = torch.full((n * T, 2), -1, dtype=torch.int32, device=DEV)
        self.rules = V.token_rules(repetition=1.1, presence=0.05, frequency=0.02, allowed=self.allowed, history=self.history,
                                   history_len=self.told, parents=self.parents, drafted=self.drafted)
        for i, t in enumerate(self.texts):                      # the prompts, one sequence at a time
            s = i32([i])
            V.vlac_pages_extend(self.p, s, 1, len(t), self.pos)
            for l in range(toy.layers):
                x = toy.qkv[l][torch.tensor(t, device=DEV)][None]
                q, k, v = x.split((toy.hq, toy.hkv, toy.hkv), 2)
                V.vlac_pages_append_rotated(self.p, l, s, self.pos, 1, len(t), toy.rot, None, toy.hq, q, k, v, torch.empty_like(q.contiguous()),
                                            *toy.gains)

    def turn(self):
        """One pass, all of it on the device."""
        toy, n, T = self.toy, self.n, self.T
        V.vlac_pages_extend(self.p, self.seqs, n, T, self.pos)
        V.vlac_attend_tree_plan(self.p, self.seqs, self.pos, n, T, toy.hq, None, self.parents, self.places, self.ws)
        for l in range(toy.layers):
            x = toy.qkv[l].index_select(0, self.drafted.reshape(-1)).view(n, T, -1, toy.hd)
            q, k, v = x.split((toy.hq, toy.hkv, toy.hkv), 2)
            V.vlac_pages_append_rotated(self.p, l, self.seqs, self.pos, n, T, toy.rot, self.places, toy.hq, q, k, v, self.q[l], *toy.gains)
            V.vlac_attend_tree(self.p, l, n, T, toy.hq, self.q[l], self.outs[l], self.ws)
        self.raw.copy_(toy.logits(self.drafted.reshape(-1), self.outs))
        V.vlac_choose_tokens(self.raw, self.rules, self.ruled, self.chosen, self.ws2)
        V.vlac_tree_accept(self.parents, self.drafted, self.chosen, n, T, self.path, self.count, self.token)
        V.vlac_pages_keep(self.p, self.seqs, self.pos, n, T, self.path, self.count)

    def give(self, parents, drafted, texts):
        self.parents.copy_(i32(parents))
        self.drafted.copy_(i32(drafted))
        self.told.copy_(i32([len(t) for t in texts]))
        for i, t in enumerate(texts):
            self.history[i, :len(t)] = i32(t)

    def state(self):
        return [x.clone() for x in (*self.p.tensors[:4], self.outs, self.places, self.ruled, self.chosen, self.path, self.count, self.token)]


def trees_for(toy, roots, T, rng, accept):
    """Trees that hold the first accept[i] tokens of what follows, among other drafts."""
    after, parents, drafted = toy.after.tolist(), [], []
    for r, a in zip(roots, accept):
        there = rng.randint(a, T)
        path = [0] + sorted(rng.sample(range(1, there), a - 1))
        par = M.tree(rng, T, "random", there)
        tok = [r] + [rng.randrange(VOCAB) for _ in range(T - 1)]
        for u, t in zip(path, path[1:]):
            par[t] = u
            tok[t] = after[tok[u]]
        for t in range(1, there):                               # nothing else that follows
            if t not in path and tok[t] == after[tok[par[t]]]:
                tok[t] = (tok[t] + 1) % VOCAB
        for t in range(1, there):                               # (changed tokens may have been parents)
            if t not in path and tok[t] == after[tok[par[t]]]:
                par[t], tok[t] = 0, (after[r] + 1) % VOCAB
        parents.append(par)
        drafted.append(tok)
    return parents, drafted


def rotated(toy, tokens):
    """Queries and keys of a text in 64 bits, [layers, N, heads, hd]."""
    import torch
    half = toy.hd // 2
    x = toy.qkv[:, torch.tensor(tokens, device=DEV)].double()
    q, k = x[:, :, :toy.hq], x[:, :, toy.hq:toy.hq + toy.hkv]
    if toy.gains[0] is not None:
        q, k = (y / torch.sqrt(y.square().mean(-1, keepdim=True) + 1e-6) * g.double() for y, g in ((q, toy.gains[0]), (k, toy.gains[1])))
    angle = 2 * math.pi * torch.arange(len(tokens), device=DEV).double()[:, None] * toy.rot.tensors[0]
    co, si = torch.cos(angle)[:, None], torch.sin(angle)[:, None]
    return [torch.cat([y[..., :half] * co - y[..., half:] * si, y[..., half:] * co + y[..., :half] * si], -1) for y in (q, k)]


def attended(toy, q, k, v):
    """The last rows of a text, in 64 bits: q [layers, m, hq, hd] over k, v [layers, N, hkv, hd]."""
    import torch
    m, N, grp = q.shape[1], k.shape[1], toy.hq // toy.hkv
    q, k, v = (y.double().transpose(1, 2) for y in (q, k.repeat_interleave(grp, 2), v.repeat_interleave(grp, 2)))
    s = q @ k.transpose(2, 3) / math.sqrt(toy.hd)
    s = s.masked_fill(torch.ones((m, N), dtype=torch.bool, device=DEV).triu(N - m + 1), -math.inf)
    return (torch.softmax(s, 3) @ v).transpose(1, 2)


LAYOUTS = [(4, 4, 64, 1, False), (12, 2, 128, 0, True), (6, 3, 64, 1, True)]


@pytest.mark.parametrize("hq,hkv,hd,operand,norm", LAYOUTS)
def test_turn_after_turn(hq, hkv, hd, operand, norm):
    import torch
    n, T, turns = 5, 13, 4
    toy = Toy(hq, hkv, hd, operand, 2, seed=hd + hq, norm=norm)
    d = Drafts(toy, n, T, 25, turns, seed=hq)
    rng = random.Random(hq)
    texts, roots = [list(t) for t in d.texts], [7, 0, 39, 12, 12]
    for turn in range(turns):
        accept = [1 + (turn + 2 * i) % 6 for i in range(n)]
        parents, drafted = trees_for(toy, roots, T, rng, accept)
        d.give(parents, drafted, texts)
        d.turn()
        assert V.vlac_pages_check(d.p, check=False) == OK
        path, count, token = d.path.tolist(), d.count.tolist(), d.token.tolist()
        assert count == accept
        assert d.chosen.tolist() == [M_first(x) for x in d.ruled.tolist()]
        after = toy.after.tolist()
        for i in range(n):
            mine = path[i][:count[i]]
            tokens = [drafted[i][t] for t in mine]
            assert token[i] == after[tokens[-1]] and d.places[i].tolist() == M.places(parents[i], len(texts[i]))
            texts[i] += tokens
            N, m = len(texts[i]), len(tokens)
            # what the cache holds now is the text's keys and values, and the queries were the path's
            assert d.p.tensors[3][i].item() == N
            data = d.p.tensors[0].view(torch.int16).view(-1, toy.layers, 2, hkv, PAGE * hd)
            row = d.p.tensors[2][i].tolist()
            k, v = (torch.stack([data[row[at // PAGE], :, w][..., torch.tensor(f(hd)[at % PAGE], device=DEV)] for at in range(N)], 1).view(toy.dt)
                    for w, f in ((0, k_tile_at), (1, v_tile_at)))
            assert torch.equal(v, toy.qkv[:, torch.tensor(texts[i], device=DEV), hq + hkv:])
            q = d.q[:, i, mine]
            for got, want in zip((q, k), rotated(toy, texts[i])):
                want = want[:, -got.shape[1]:]
                assert bool(((got.double() - want).abs() <= toy.step * want.abs() + toy.kq).all())
            want = toy.logits(i32(tokens), attended(toy, q, k, v))
            off = (d.raw.view(n, T, VOCAB)[i, mine] - want).abs().max().item()
            assert off <= toy.tol, (off, toy.tol)
        roots = token
    V.vlac_pages_free(d.p, d.seqs, n)
    assert not bool(d.p.tensors[1].any()) and V.vlac_pages_check(d.p, check=False) == OK


def M_first(x):
    return max(range(len(x)), key=lambda i: (x[i], -i)) if max(x) > -math.inf else -1


def script(toy, d, turns, seed):
    """The turns' inputs, made beforehand: what the turns accept is known."""
    rng, after = random.Random(seed), toy.after.tolist()
    texts, roots, out = [list(t) for t in d.texts], [rng.randrange(VOCAB) for _ in range(d.n)], []
    for turn in range(turns):
        accept = [1 + (turn + i) % 5 for i in range(d.n)]
        parents, drafted = trees_for(toy, roots, d.T, rng, accept)
        out.append((parents, drafted, [list(t) for t in texts]))
        for i, a in enumerate(accept):
            for _ in range(a):
                texts[i].append(roots[i])
                roots[i] = after[roots[i]]
    return out


def same(a, b):
    import torch
    return all(torch.equal(x.view(torch.int16) if x.is_floating_point() and x.element_size() == 2 else x,
                           y.view(torch.int16) if y.is_floating_point() and y.element_size() == 2 else y) for x, y in zip(a, b))


def test_a_turn_as_a_graph():
    """Captured once and replayed turn after turn, eager turns of another batch in between: the same bits as eager turns."""
    import torch
    toy = Toy(8, 2, 64, 1, 2, seed=1, norm=True)
    turns = 6
    eager, graphed, other = (Drafts(toy, 3, 9, 40, turns + 2, seed=4) for _ in range(3))
    inputs = script(toy, eager, turns, 9)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):                             # (libraries warm up on a batch that nobody looks at)
        warm = Drafts(toy, 3, 9, 40, 2, seed=4)
        warm.give(*inputs[0])
        warm.turn()
    torch.cuda.current_stream().wait_stream(stream)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        graphed.turn()
    for turn in range(turns):
        eager.give(*inputs[turn])
        eager.turn()
        graphed.give(*inputs[turn])
        graph.replay()
        if turn % 2:
            torch.cuda.synchronize()
            other.give(*inputs[0])
            other.turn()
        assert same(eager.state(), graphed.state()), turn
        assert V.vlac_pages_check(graphed.p, check=False) == OK


def test_two_pools_on_two_streams():
    import torch
    toy = Toy(12, 2, 128, 0, 2, seed=2, norm=False)
    turns = 4
    want, got = [[Drafts(toy, 4, 17, 300, turns, seed=s) for s in (5, 6)] for _ in range(2)]
    inputs = [script(toy, d, turns, 3 + k) for k, d in enumerate(want)]
    for k, d in enumerate(want):
        for x in inputs[k]:
            d.give(*x)
            d.turn()
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for turn in range(turns):
        for k, d in enumerate(got):
            with torch.cuda.stream(streams[k]):
                d.give(*inputs[k][turn])
                d.turn()
    torch.cuda.synchronize()
    for a, b in zip(want, got):
        assert same(a.state(), b.state())


def test_a_stream_by_argument():
    """Every call on a stream that is not the current one."""
    import torch
    toy = Toy(4, 4, 64, 1, 1, seed=3, norm=False)
    a, b = (Drafts(toy, 2, 6, 20, 1, seed=8) for _ in range(2))
    x = script(toy, a, 1, 2)[0]
    a.give(*x)
    a.turn()
    b.give(*x)
    rows = toy.qkv[0].index_select(0, b.drafted.reshape(-1)).view(2, 6, -1, 64)
    q, k, v = rows.split((4, 4, 4), 2)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    on = dict(stream=s)
    V.vlac_pages_extend(b.p, b.seqs, 2, 6, b.pos, **on)
    V.vlac_attend_tree_plan(b.p, b.seqs, b.pos, 2, 6, 4, None, b.parents, b.places, b.ws, **on)
    V.vlac_pages_append_rotated(b.p, 0, b.seqs, b.pos, 2, 6, toy.rot, b.places, 4, q, k, v, q, None, None, **on)
    V.vlac_attend_tree(b.p, 0, 2, 6, 4, q, b.outs[0], b.ws, **on)
    s.synchronize()
    b.raw.copy_(toy.logits(b.drafted.reshape(-1), b.outs))
    torch.cuda.synchronize()
    V.vlac_choose_tokens(b.raw, b.rules, b.ruled, b.chosen, b.ws2, **on)
    V.vlac_tree_accept(b.parents, b.drafted, b.chosen, 2, 6, b.path, b.count, b.token, **on)
    V.vlac_pages_keep(b.p, b.seqs, b.pos, 2, 6, b.path, b.count, **on)
    s.synchronize()
    assert same(a.state(), b.state())
