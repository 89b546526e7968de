"""Answers written with drafted tokens: products with 4-bit weights, keys and values appended with their turns, attention of
the trees, a token after each node, and the accepted path kept, as a user's loop has them, on a small model of two layers."""
import math

import numpy as np
import pytest
import torch

import paper_2306_10015_gb300 as jb

pytestmark = pytest.mark.gpu

I32 = dict(dtype=torch.int32, device="cuda")
D, HEADS, KV_HEADS, WIDTH, VOCAB, LAYERS = 64, 4, 2, 256, 500, 2
KINDS = ("q", "k", "v", "o")


def i32(v):
    return torch.tensor(v, **I32)


class Model:
    """h = emb[token]; per layer h += o(attention(turned q, turned k, v)); logits = head(h) of the normalised h."""

    def __init__(self, dtype, seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.dtype = dtype
        self.shapes = [(HEADS * D if kind == "q" else WIDTH if kind == "o" else KV_HEADS * D, HEADS * D if kind == "o" else WIDTH)
                       for _ in range(LAYERS) for kind in KINDS] + [(VOCAB, WIDTH)]
        tensors = []
        for out, inner in self.shapes:
            codes = torch.randint(0, 256, (out * inner // 2,), dtype=torch.uint8, device="cuda", generator=g)
            scale = (torch.rand(out * inner // 64, device="cuda", generator=g) + 0.5) * (2 / math.sqrt(inner))
            tensors.append((codes, scale, out * inner))
        self.table = jb.Q4Table(tensors)
        self.emb = torch.randn(VOCAB, WIDTH, device="cuda", generator=g).to(dtype)
        self.rotation = jb.Rotation.powers(D)
        self.freq = torch.from_numpy(10000.0 ** (-np.arange(0, D, 2) / D)).cuda()

    def product(self, i, x):
        return jb.jb_q4_matmul(self.table, i, x, self.shapes[i][0])

    def norm(self, h):
        return h * torch.rsqrt(h.square().mean(-1, keepdim=True) + 1e-6)

    def nodes(self, cache, tokens, rows, pos, turns, attend):
        """Logits after each of the tokens; attend(layer, q) has the attention."""
        h = self.emb[tokens.long()]
        for i in range(LAYERS):
            x = self.norm(h)
            q, k, v = (self.product(4 * i + j, x).view(len(tokens), -1, D) for j in range(3))
            q = jb.jb_cache_append(cache, i, q, k, v, rows, pos, self.rotation, turns=turns)
            h = h + self.product(4 * i + 3, attend(i, q).view(len(tokens), -1))
        return self.product(4 * LAYERS, self.norm(h))

    def plain(self, tokens):
        """The same formulas in 64 bits: logits after each token of one sequence."""
        levels = torch.from_numpy(jb.jb_q4_levels().astype(np.float64)).cuda()

        def product(i, x):
            codes, scale, n = self.table.tensors[i]
            w = levels[torch.stack([codes & 15, codes >> 4], -1).view(-1).long()] * scale.double().repeat_interleave(64)
            return x @ w.view(self.shapes[i]).T

        def turned(x):
            a = torch.arange(len(tokens), device="cuda").double()[:, None, None] * self.freq
            lo, hi = x[..., :D // 2], x[..., D // 2:]
            return torch.cat([lo * a.cos() - hi * a.sin(), hi * a.cos() + lo * a.sin()], -1)

        n = len(tokens)
        h = self.emb[torch.tensor(tokens, device="cuda")].double()
        mask = torch.ones(n, n, dtype=torch.bool, device="cuda").tril()
        for i in range(LAYERS):
            x = self.norm(h)
            q, k, v = (product(4 * i + j, x).view(n, -1, D) for j in range(3))
            q, k = turned(q), turned(k).repeat_interleave(HEADS // KV_HEADS, 1)
            s = torch.einsum("ihd,jhd->hij", q, k) / math.sqrt(D)
            w = torch.softmax(s.masked_fill(~mask, -math.inf), -1)
            o = torch.einsum("hij,jhd->ihd", w, v.repeat_interleave(HEADS // KV_HEADS, 1))
            h = h + product(4 * i + 3, o.reshape(n, -1))
        return product(4 * LAYERS, self.norm(h))


def cache_of(dtype, rows=4, pages=80):
    table = jb.PageTable.empty(rows, 20, pages, 16)
    kv = [torch.full((pages, KV_HEADS, 16, D), float("nan"), dtype=dtype, device="cuda") for _ in range(2 * LAYERS)]
    return jb.KVCache(table, kv[:LAYERS], kv[LAYERS:])


def draft_step(model, cache, trees, tokens, row_of, index, depth, counts, status):
    """Room for the trees' nodes, the model over them, and a token after each node."""
    base = cache.pages.lens[row_of.long()]
    jb.jb_cache_reserve(cache, trees.rows, counts, status=status)
    logits = model.nodes(cache, tokens, row_of, base + index, base + depth, lambda i, q: jb.jb_attend_tree(cache, i, q, trees))
    return logits, jb.jb_sample(logits, torch.zeros(len(tokens), **I32), temperature=0.0)[0]


def random_trees(rng, rows, most):
    starts, parents = [0], []
    for _ in rows:
        n = int(rng.integers(1, most + 1))
        parents += [-1] + [int(rng.integers(max(0, j - 5), j)) for j in range(1, n)]
        starts.append(starts[-1] + n)
    return starts, parents


def shape_of(rows, starts, parents):
    row_of, index, depth = [], [], []
    for i, r in enumerate(rows):
        for j in range(starts[i + 1] - starts[i]):
            p = parents[starts[i] + j]
            depth.append(0 if p < 0 else depth[starts[i] + p] + 1)
            row_of.append(r)
            index.append(j)
    return row_of, index, depth


# Weights have a mean size of 0.07, so a product of 256 terms has rows of norm 1.3, and it is off by less than (256 / 16 + 73)
# 2^-22 of sum |x w| ~ 14 (the products' own tolerance): 3e-4. With every product that far off, and errors that do not line up:
# scores by 3e-4 |q| sqrt(2) / 8 ~ 5e-4 (|q| ~ 10), weights by twice that of themselves, outputs of size 1.3 by 2e-3; the second
# layer's inputs by 2e-3, its scores by 5e-3, its outputs by 1e-2; a logit by 1.3 times that, and the farthest of some thousands
# by four times as much. A wrong mask, turn, page or path moves logits by their size, 1.3 and more.
WORST = 0.05


def test_drafted_tokens_are_those_of_the_whole_sequence():
    rng = np.random.default_rng(5)
    model, cache = Model(torch.float32), cache_of(torch.float32)
    rows = [2, 0, 3]
    said = {r: [int(t) for t in rng.integers(0, VOCAB, n)] for r, n in zip(rows, (37, 1, 90))}
    after = {}
    for r in rows:                      # the prompts: chains
        n = len(said[r])
        trees = jb.DraftTrees(i32([r]), i32([0, n]), i32(list(range(-1, n - 1))))
        logits, tokens = draft_step(model, cache, trees, i32(said[r]), i32([r] * n), i32(list(range(n))), i32(list(range(n))),
                                    i32([n]), torch.ones(1, **I32))
        assert (logits.double() - model.plain(said[r])).abs().max() <= WORST
        after[r] = int(tokens[-1])
    assert cache.pages.lens.tolist() == [1, 0, 37, 90]
    for turn in range(6):
        starts, parents = random_trees(rng, rows, 40 if turn != 3 else 1)
        drafted = [int(t) for t in rng.integers(0, VOCAB, starts[-1])]
        for i, r in enumerate(rows):
            drafted[starts[i]] = after[r]
        row_of, index, depth = shape_of(rows, starts, parents)
        trees = jb.DraftTrees(i32(rows), i32(starts), i32(parents))
        status = torch.ones(1, **I32)
        logits, tokens = draft_step(model, cache, trees, i32(drafted), i32(row_of), i32(index), i32(depth),
                                    i32(np.diff(starts).tolist()), status)
        assert status.item() == 0
        leaves, tokens = [], tokens.tolist()
        for i, r in enumerate(rows):
            path_of = {}
            for j in range(starts[i + 1] - starts[i]):
                p = parents[starts[i] + j]
                path_of[j] = (path_of[p] if p >= 0 else []) + [drafted[starts[i] + j]]
            for j, path in path_of.items():
                want = model.plain(said[r] + path)[-1]
                assert (logits[starts[i] + j].double() - want).abs().max() <= WORST, (turn, r, j)
            leaf = int(rng.integers(0, len(path_of)))       # as if the drafts of one path were all right
            leaves.append(leaf)
            said[r] += path_of[leaf]
            after[r] = tokens[starts[i] + leaf]
        assert jb.jb_cache_keep(cache, trees, i32(leaves)).item() == 0
        assert cache.pages.lens.tolist() == [len(said.get(r, [])) for r in range(4)]
        assert int((cache.pages.refs > 0).sum()) == sum(-(-len(s) // 16) for s in said.values())
    # One token each by the attention that was there before, over what the drafts left in the cache.
    base = cache.pages.lens[i32(rows).long()].clone()
    jb.jb_cache_reserve(cache, i32(rows), i32([1] * 3))
    logits = model.nodes(cache, i32([after[r] for r in rows]), i32(rows), base, None,
                         lambda i, q: jb.jb_attend(cache, i, q, i32(rows), base))
    for i, r in enumerate(rows):
        assert (logits[i].double() - model.plain(said[r] + [after[r]])[-1]).abs().max() <= WORST


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_graphs_of_whole_steps(dtype):
    """Two captured graphs of one cache and one table of weights, replayed in turn on two streams, against the same calls made
    one by one: every token, logit, table and page."""
    rng = np.random.default_rng(9)
    model = Model(dtype)
    shapes = []
    for rows in ([1, 3], [0, 2, 1]):
        starts, parents = random_trees(rng, rows, 60)
        shapes.append((rows, starts, parents))

    def make():
        cache = cache_of(dtype)
        assert jb.jb_cache_reserve(cache, i32([0, 1, 2, 3]), i32([21, 16, 1, 47])).item() == 0
        g = torch.Generator(device="cuda").manual_seed(2)
        n = 85
        kv = [torch.randn(n, KV_HEADS, D, generator=g, device="cuda").to(dtype) for _ in range(2)]
        rows = [0] * 21 + [1] * 16 + [2] + [3] * 47
        pos = list(range(21)) + list(range(16)) + [0] + list(range(47))
        for i in range(LAYERS):
            jb.jb_cache_write(cache, i, kv[0], kv[1], i32(rows), i32(pos))
        steps = []
        for rows, starts, parents in shapes:
            row_of, index, depth = (i32(v) for v in shape_of(rows, starts, parents))
            steps.append(dict(trees=jb.DraftTrees(i32(rows), i32(starts), i32(parents)), tokens=torch.zeros(starts[-1], **I32),
                              row_of=row_of, index=index, depth=depth, counts=i32(np.diff(starts).tolist()),
                              status=torch.ones(1, **I32), kept=torch.ones(1, **I32), leaves=torch.zeros(len(rows), **I32)))
        return cache, steps

    def run(cache, s, leaves=True):
        logits, tokens = draft_step(model, cache, s["trees"], s["tokens"], s["row_of"], s["index"], s["depth"], s["counts"], s["status"])
        if leaves:
            jb.jb_cache_keep(cache, s["trees"], s["leaves"], status=s["kept"])
        return logits, tokens

    spare, eager, captured = make(), make(), make()
    for s in spare[1]:
        run(spare[0], s)
    (eager, es), (captured, cs) = eager, captured
    graphs, outs = [], []
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for s, stream in zip(cs, streams):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            outs.append(run(captured, s))
        graphs.append(graph)
    for turn in range(8):
        which = turn % 2
        rows, starts, parents = shapes[which]
        tokens = torch.randint(0, VOCAB, (starts[-1],), **I32)
        leaves = i32([int(rng.integers(-1, min(9, b - a))) for a, b in zip(starts, starts[1:])])
        for s in (es[which], cs[which]):
            s["tokens"].copy_(tokens)
            s["leaves"].copy_(leaves)
        want = run(eager, es[which])
        torch.cuda.synchronize()
        with torch.cuda.stream(streams[which]):
            graphs[which].replay()
        torch.cuda.synchronize()
        assert es[which]["status"].item() == cs[which]["status"].item() == 0
        assert es[which]["kept"].item() == cs[which]["kept"].item() == 0
        assert torch.equal(want[0], outs[which][0]) and torch.equal(want[1], outs[which][1]), turn
        assert torch.isfinite(want[0]).all()
        for a, b in zip((eager.pages.table, eager.pages.lens, eager.pages.refs), (captured.pages.table, captured.pages.lens, captured.pages.refs)):
            assert torch.equal(a, b)
        for r, n in enumerate(eager.pages.lens.tolist()):
            ids = eager.pages.table[r, :-(-n // 16)].long()
            for a, b in zip(eager.keys + eager.values, captured.keys + captured.values):
                assert torch.equal(a[ids].transpose(1, 2).reshape(-1, KV_HEADS, D)[:n], b[ids].transpose(1, 2).reshape(-1, KV_HEADS, D)[:n])
