"""What a decoder needs to write answers from drafted tokens, as cases that can be timed and compared.

A forward-only method spends its steps writing answers. Several tokens of an answer can be checked in one pass over
the weights and the cache: a tree of drafted tokens is appended to its row, attended to at once, and the path that
the model would have written itself is kept. The weights may be the 4-bit ones that jb_perturb_q4 perturbs.

* ``append``  queries and keys turned by their positions, keys and values to their places in the pages;
* ``tree``    each drafted token against its row's tokens and its own ancestors;
* ``keep``    the path to one drafted token stays, the others' places are given back and reserved for the next tree;
* ``q4``      products of a few rows with a matrix of 4-bit codes and a scale per 64 of them.

``prepare`` makes the inputs from the seed, ``run`` makes the calls (``own``) or computes the same in elementary torch
operations, ``exact`` restates them in 64 bits, row by row.
"""
from __future__ import annotations

import math
from statistics import NormalDist

import numpy as np
import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "bf16": 2}


def listed():
    return [
        # One token of a small fp32 decoder (12 heads of 64): a call's latency is all.
        dict(name="append-1-f32", op="append", dtype="f32", n=1, rows=1, heads=12, group=1, d=64, dims=64, pairs="half", far=0, page=16,
             layout="hnd", lo=37, hi=37, sizes_seed=10),
        # The drafted tokens of 48 rows, far into a long text whose beginning the cache no longer holds; four query heads
        # to a key head.
        dict(name="append-337-far-bf16", op="append", dtype="bf16", n=337, rows=48, heads=8, group=4, d=128, dims=128, pairs="half",
             far=1_000_003, page=16, layout="hnd", lo=65, hi=2000, sizes_seed=11),
        # The tokens of a batch of prompts on the shape of the 6.7B decoder; neighbours are turned, half of each head.
        dict(name="append-8191-bf16", op="append", dtype="bf16", n=8191, rows=8, heads=32, group=1, d=128, dims=64, pairs="next", far=0, page=32,
             layout="nhd", lo=1, hi=9, sizes_seed=12),
        # Five drafted tokens of one short fp32 answer.
        dict(name="tree-1x5-f32", op="tree", dtype="f32", n=1, tlo=5, thi=5, shape="near", heads=12, group=1, d=64, page=16, layout="hnd", lo=37, hi=37,
             sizes_seed=0, empty=0, window=0, softcap=0.0, bias=False),
        # A batch of ragged answers on the shape of the 6.7B decoder, trees of up to 33 tokens, a finished row among them.
        dict(name="tree-24-ragged-bf16", op="tree", dtype="bf16", n=24, tlo=2, thi=33, shape="wide", heads=32, group=1, d=128, page=16, layout="hnd",
             lo=65, hi=2000, sizes_seed=1, empty=1, window=0, softcap=0.0, bias=False),
        # Three rows over very long contexts, eight query heads to a key head, scores capped.
        dict(name="tree-3-long-g8-bf16", op="tree", dtype="bf16", n=3, tlo=50, thi=64, shape="near", heads=8, group=8, d=128, page=64, layout="nhd",
             lo=50001, hi=65000, sizes_seed=2, empty=0, window=0, softcap=30.0, bias=False),
        # Chains: the next 255 tokens of 16 prompts on the shape of the 13B decoder (40 heads of 128).
        dict(name="tree-16x255-chain-bf16", op="tree", dtype="bf16", n=16, tlo=255, thi=255, shape="chain", heads=40, group=1, d=128, page=32, layout="hnd",
             lo=400, hi=1793, sizes_seed=3, empty=0, window=0, softcap=0.0, bias=False),
        # Three small trees, 12 layers of a small fp32 decoder.
        dict(name="keep-3-f32", op="keep", dtype="f32", n=3, tlo=4, thi=7, shape="near", heads=12, d=64, page=16, layout="hnd", layers=12, lo=20, hi=90,
             sizes_seed=4),
        # 64 answers on the shape of the 1.3B decoder (24 layers of 32 heads of 64), trees of up to 64 tokens.
        dict(name="keep-64-bf16", op="keep", dtype="bf16", n=64, tlo=33, thi=64, shape="near", heads=32, d=64, page=16, layout="nhd", layers=24, lo=65, hi=400,
             sizes_seed=5),
        # A projection of a small decoder for one fp32 token.
        dict(name="q4-1x768-f32", op="q4", dtype="f32", n=1, out=768, inner=768, bias=True),
        # The first matrix of the 13B decoder's network for one token: reading the codes is all.
        dict(name="q4-1-fc1-13b-bf16", op="q4", dtype="bf16", n=1, out=20480, inner=5120, bias=False),
        # Its second matrix for 17 drafted tokens.
        dict(name="q4-17-fc2-13b-bf16", op="q4", dtype="bf16", n=17, out=5120, inner=20480, bias=True),
    ]


def draw(rng):
    """One more case: every operation, type and layout, sizes spread over their logarithm."""
    def log_uniform(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    op = rng.choice(["append", "append", "tree", "tree", "tree", "keep", "q4", "q4"])
    case = dict(op=op, dtype=rng.choice(["f32", "bf16", "bf16"]))
    if op == "q4":
        case.update(n=log_uniform(1, 64), out=log_uniform(64, 28672), bias=rng.random() < 0.5)
        case["inner"] = 64 * log_uniform(1, min(320, int(1.1e8 / case["out"] / 64)))
        return case
    case.update(page=rng.choice([16, 16, 32, 48, 64, 128]), layout=rng.choice(["hnd", "nhd"]), d=rng.choice([64, 64, 80, 96, 128, 128, 256]),
                sizes_seed=rng.randrange(1 << 30))
    if op == "append":
        case.update(n=log_uniform(1, 8192), heads=log_uniform(1, 32), group=rng.choice([1, 1, 2, 4, 5, 8]), lo=1, hi=log_uniform(1, 1000),
                    pairs=rng.choice(["half", "next"]), far=rng.choice([0, 0, log_uniform(1000, 1 << 30)]))
        case["n"] = min(case["n"], int(2.2e8 / (case["heads"] * (2 * case["group"] + 4) * case["d"])) + 1)
        case.update(rows=min(case["n"], log_uniform(1, 256)), dims=rng.choice([case["d"], case["d"], case["d"] // 2, 32]))
        return case
    case.update(n=log_uniform(1, 64), shape=rng.choice(["near", "near", "wide", "chain"]), thi=log_uniform(1, 256))
    case["tlo"] = rng.choice([1, max(1, case["thi"] // 2), case["thi"]])
    if op == "tree":
        case["group"] = rng.choice([1, 1, 2, 4, 5, 8, 16])
        case["heads"] = min(log_uniform(1, 40), max(1, 128 // case["group"]))
        token = case["n"] * case["heads"] * case["d"]
        # bytes, operations and the plain form's scores of a row's tokens
        most = min(7e8 / (2 * SIZE[case["dtype"]] * token), 3.5e11 / (4.0 * token * case["group"] * case["thi"]),
                   6e8 / (case["n"] * case["heads"] * case["group"] * case["thi"]), 4e8 / token)
        if case["dtype"] == "f32":
            most = min(most, 4e10 / (4.0 * token * case["group"] * case["thi"]))
        case["hi"] = log_uniform(1, max(2, min(100_000, int(most) - case["thi"])))
        case["lo"] = rng.choice([1, max(1, case["hi"] // 2), case["hi"]])
        case.update(empty=rng.choice([0, 1]) if case["n"] > 1 else 0, window=rng.choice([0, 0, log_uniform(1, 4096)]), softcap=rng.choice([0.0, 0.0, 30.0]),
                    bias=rng.random() < 0.3)
        return case
    case.update(thi=min(case["thi"], 128), heads=log_uniform(1, 32), layers=log_uniform(1, 24))
    case["tlo"] = min(case["tlo"], case["thi"])
    token = 2 * case["layers"] * case["heads"] * case["d"] * SIZE[case["dtype"]]
    case["hi"] = log_uniform(1, max(2, min(2048, int(4e9 / token / case["n"]) - case["thi"] - 2 * case["page"])))
    case["lo"] = max(1, case["hi"] // 4)
    return case


# --- shapes -------------------------------------------------------------------------------

def _spread(g, lo, hi, n):
    """n sizes, spread over their logarithm, the first the largest."""
    v = np.exp(g.uniform(math.log(lo), math.log(hi + 1), size=n)).astype(np.int64).clip(lo, hi)
    v[0] = hi
    return v


def _pages(lens, page):
    return -(-lens // page)


def _trees(case):
    """Tokens that the rows have, drafted tokens of each, and the drafted tokens' parents within their tree."""
    g = np.random.default_rng(case["sizes_seed"])
    had, size = _spread(g, case["lo"], case["hi"], case["n"]), _spread(g, case["tlo"], case["thi"], case["n"])
    if case.get("empty"):
        size[case["n"] // 2] = 0
    parents = []
    for t in size.tolist():
        j = np.arange(t)
        back = np.minimum(g.geometric(0.6, size=t) - 1, 3)
        p = {"chain": j - 1, "wide": np.where(j > 0, (j - 1) // 3, -1), "near": np.where(j > 0, np.maximum(j - 1 - back, 0), -1)}[case["shape"]]
        parents.append(p)
    return had, size, parents


def _depths(parents):
    d = np.zeros(len(parents), dtype=np.int64)
    for j, p in enumerate(parents):
        d[j] = d[p] + 1 if p >= 0 else 0
    return d


def _leaves(case):
    """The drafted token of each tree whose path is kept."""
    g = np.random.default_rng([case["sizes_seed"], 1])
    _, size, _ = _trees(case)
    return (g.random(case["n"]) * size).astype(np.int64)


def _steps(dims):
    """The turn of each pair per position, in 2^-64 of a full turn: 10000^(-2i / dims) radians."""
    f = np.float64(10000.0) ** (-2.0 * np.arange(dims // 2) / dims) / (2 * math.pi)
    return (f * 2.0**64).astype(np.uint64).view(np.int64)


def _levels():
    """The 16 levels of the 4-bit code."""
    q, d = NormalDist().inv_cdf, 1 / 32
    v = np.array([q(d + (0.5 - d) * j / 7) for j in range(7)] + [0.0] + [q(0.5 + (0.5 - d) * j / 8) for j in range(1, 9)])
    return (v / np.abs(v).max()).astype(np.float32)


def _pool(case, n_pages, layers, gen):
    """Keys and values [2 layers, pages, heads, tokens, d], N(0, 1), in memory by heads or by tokens."""
    h, p, d = case["heads"], case["page"], case["d"]
    shape = (2 * layers, n_pages, h, p, d) if case["layout"] == "hnd" else (2 * layers, n_pages, p, h, d)
    x = torch.empty(shape, dtype=DTYPES[case["dtype"]], device="cuda").normal_(generator=gen)
    return x if case["layout"] == "hnd" else x.transpose(2, 3)


def _table(lens, case, n_pages, row_pages, g):
    """Page ids of rows of these lengths in a random order, and their references."""
    table = np.full((len(lens), row_pages), -1, dtype=np.int32)
    need = _pages(lens, case["page"])
    ids = g.permutation(n_pages)[:int(need.sum())].astype(np.int32)
    table[np.arange(row_pages)[None, :] < need[:, None]] = ids
    refs = np.zeros(n_pages, dtype=np.int32)
    refs[ids] = 1
    return table, refs


def _cuda(a, dtype=None):
    return torch.from_numpy(np.ascontiguousarray(a)).to("cuda", dtype=dtype)


def prepare(case, seed):
    g = np.random.default_rng([seed, 7])
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed + 1)
    s, op, dtype, i32 = dict(case=case), case["op"], DTYPES[case["dtype"]], torch.int32
    if op == "q4":
        out, inner, n = case["out"], case["inner"], case["n"]
        s["codes"] = torch.randint(0, 256, (out * inner // 2,), dtype=torch.uint8, device="cuda", generator=gen)
        s["scale"] = 0.02 + 0.03 * torch.rand(out * inner // 64, device="cuda", generator=gen)
        x = torch.randn(n, inner, device="cuda", generator=gen)
        x[:, torch.rand(inner, device="cuda", generator=gen) < 0.002] *= 60.0  # some channels stand out
        s["x"] = x.to(dtype)
        s["bias"] = torch.randn(out, device="cuda", generator=gen).to(dtype) if case["bias"] else None
        s["levels"] = _cuda(_levels())
        if own:
            import paper_2306_10015_gb300 as jb
            s["weights"] = jb.Q4Table([(s["codes"], s["scale"], out * inner)])
        return s
    page, layers, h, d = case["page"], case.get("layers", 1), case["heads"], case["d"]
    if op == "append":
        # each row's share of the n tokens, after the tokens that it has
        n = case["n"]
        had, new = _spread(np.random.default_rng(case["sizes_seed"]), case["lo"], case["hi"], case["rows"]), np.diff(np.arange(case["rows"] + 1) * n // case["rows"])
        lens = had + new
        rows = np.repeat(np.arange(case["rows"]), new)
        s["rows"] = _cuda(rows, i32)
        s["pos"] = _cuda(had[rows] + np.arange(n) - (np.cumsum(new) - new)[rows], i32)
        s["turns"] = s["pos"] + case["far"]
        qh = h * case["group"]
        qkv = torch.randn(n, (qh + 2 * h) * d, device="cuda", generator=gen).to(dtype)  # as the projection leaves them
        s["q"], s["new_k"], s["new_v"] = (x.view(n, -1, d) for x in qkv.split([qh * d, h * d, h * d], 1))
        s["steps"] = _cuda(_steps(case["dims"]))
    else:
        had, size, parents = _trees(case)
        lens = had + size
        s["trees"] = torch.arange(case["n"], dtype=i32, device="cuda")
        s["starts"] = _cuda(np.concatenate([[0], np.cumsum(size)]), i32)
        s["parents"] = _cuda(np.concatenate(parents), i32)
        if op == "tree":
            n, qh = int(size.sum()), h * case["group"]
            qkv = torch.randn(n, (qh + 2 * h) * d, device="cuda", generator=gen)
            qkv[:, :qh * d] *= 2.5  # some tokens stand out
            s["q"] = qkv.to(dtype)[:, :qh * d].view(n, qh, d)
            s["slopes"] = (2.0 ** -torch.linspace(1, 8, qh, device="cuda")).float() if case["bias"] else None
        else:
            leaves = _leaves(case)
            s["leaves"] = _cuda(leaves, i32)
            # what the next tree needs for as many tokens as this one had
            s["again"] = _cuda(size - np.array([_depths(p)[j] + 1 for p, j in zip(parents, leaves)]), i32)
    row_pages, n_pages = int(_pages(lens, page).max()) + 1, int(_pages(lens, page).sum()) + 3
    table, refs = _table(lens, case, n_pages, row_pages, g)
    s["pool"] = _pool(case, n_pages, layers, gen)
    s["table"], s["refs"], s["lens"] = _cuda(table), _cuda(refs), _cuda(lens, i32)
    s["status"] = torch.zeros(2, dtype=i32, device="cuda")
    if own:
        import paper_2306_10015_gb300 as jb
        s["cache"] = jb.KVCache(jb.PageTable(s["table"], s["lens"], s["refs"], page), list(s["pool"][:layers]), list(s["pool"][layers:]))
        if op == "append":
            s["rotation"] = jb.Rotation(s["steps"], interleaved=case["pairs"] == "next")
        else:
            s["draft"] = jb.DraftTrees(s["trees"], s["starts"], s["parents"])
    return s


# --- one pass -------------------------------------------------------------------------------

def run(state):
    op = state["case"]["op"]
    return (_run_own if own else _run_plain)[op](state)


def _own_append(s):
    import paper_2306_10015_gb300 as jb
    q = jb.jb_cache_append(s["cache"], 0, s["q"], s["new_k"], s["new_v"], s["rows"], s["pos"], s["rotation"], turns=s["turns"])
    return [q, s["pool"]]


def _own_tree(s):
    import paper_2306_10015_gb300 as jb
    c = s["case"]
    return jb.jb_attend_tree(s["cache"], 0, s["q"], s["draft"], softcap=c["softcap"], window=c["window"], slopes=s["slopes"])


def _own_keep(s):
    import paper_2306_10015_gb300 as jb
    jb.jb_cache_keep(s["cache"], s["draft"], s["leaves"], status=s["status"][:1])
    jb.jb_cache_reserve(s["cache"], s["trees"], s["again"], status=s["status"][1:])
    return [s["table"], s["lens"], s["refs"], s["status"], s["pool"]]


def _own_q4(s):
    import paper_2306_10015_gb300 as jb
    return jb.jb_q4_matmul(s["weights"], 0, s["x"], s["case"]["out"], bias=s["bias"])


def _turned(x, cos, sin, dims, pairs):
    """[n, heads, d] in 32 bits, pairs of the first `dims` elements turned, in the given type."""
    y = x.float()
    a, b = (y[..., :dims // 2], y[..., dims // 2:dims]) if pairs == "half" else (y[..., 0:dims:2], y[..., 1:dims:2])
    a, b = a * cos - b * sin, b * cos + a * sin
    front = torch.cat([a, b], -1) if pairs == "half" else torch.stack([a, b], -1).flatten(-2)
    return torch.cat([front, y[..., dims:]], -1).to(x.dtype)


def _plain_append(s):
    c, page = s["case"], s["case"]["page"]
    # whole turns fall off the 64-bit product
    angle = (s["turns"].long()[:, None] * s["steps"][None, :]).double() * (2 * math.pi / 2.0**64)
    cos, sin = torch.cos(angle).float()[:, None, :], torch.sin(angle).float()[:, None, :]
    pos = s["pos"].long()
    at = s["table"][s["rows"].long(), pos // page].long()
    s["pool"][0][at, :, pos % page, :] = _turned(s["new_k"], cos, sin, c["dims"], c["pairs"])
    s["pool"][1][at, :, pos % page, :] = s["new_v"]
    return [_turned(s["q"], cos, sin, c["dims"], c["pairs"]), s["pool"]]


def _grid(s, most):
    """Trees as [n, most]: whether there is such a node, its index among all, who is its ancestor or itself, its depth."""
    starts, parents = s["starts"].long(), s["parents"].long()
    j = torch.arange(most, device="cuda")
    real = j[None, :] < (starts[1:] - starts[:-1])[:, None]
    index = (starts[:-1, None] + j).clamp(max=parents.numel() - 1)
    parent = torch.where(real, parents[index], torch.full_like(index, -1))
    step = (j[None, None, :] == parent[:, :, None]).double() + torch.eye(most, dtype=torch.float64, device="cuda")
    up = torch.linalg.matrix_power(step, most) > 0  # paths of up to `most` steps: counts, below 2^256
    return real, index, up, up.sum(-1) - 1


def _plain_tree(s):
    c = s["case"]
    n, h, g, d, page, most = c["n"], c["heads"], c["group"], c["d"], c["page"], c["thi"]
    real, index, up, depth = _grid(s, most)
    rows = s["trees"].long()
    table = s["table"][rows].long().clamp(min=0)
    span = table.shape[1] * page
    k, v = (x[table].permute(0, 2, 1, 3, 4).reshape(n, h, span, d).float() for x in s["pool"])
    q = s["q"][index].view(n, most, h, g, d).permute(0, 2, 3, 1, 4).float()  # [n, h, g, most, d]
    x = torch.matmul(q.reshape(n, h, g * most, d), k.transpose(-1, -2)).view(n, h, g, most, span) * (1.0 / math.sqrt(d))
    if c["softcap"]:
        x = c["softcap"] * torch.tanh(x / c["softcap"])
    size = real.sum(-1)
    base = s["lens"].long()[rows] - size
    t = torch.arange(span, device="cuda")
    node = t[None, :] - base[:, None]  # the place's drafted token; before them below 0
    inside = (node >= 0) & (node < size[:, None])
    node = node.clamp(0, most - 1)
    where = torch.where(inside, base[:, None] + torch.gather(depth, 1, node), t[None, :])  # positions as a chain would have them
    back = where[:, None, :] - (base[:, None] + depth)[:, :, None]  # [n, most, span], at most 0 where seen
    seen = (t[None, :] < base[:, None])[:, None, :] | (inside[:, None, :] & torch.gather(up, 2, node[:, None, :].expand(n, most, span)))
    seen = seen & real[:, :, None]
    if c["window"]:
        seen = seen & (back > -c["window"])
    if c["bias"]:
        x = x + s["slopes"].view(1, h, g, 1, 1) * back[:, None, None].float()
    seen = seen[:, None, None]
    top = torch.where(seen, x, torch.full_like(x, -3e38)).amax(-1, keepdim=True)
    e = torch.where(seen, torch.exp(x - top), torch.zeros_like(x))
    out = torch.matmul(e.view(n, h, g * most, span), v).view(n, h, g, most, d) / e.sum(-1, keepdim=True).clamp(min=1e-30)
    return out.permute(0, 3, 1, 2, 4).reshape(n, most, h * g, d)[real].to(s["q"].dtype)


def _plain_keep(s):
    c, table, refs, lens, pool = s["case"], s["table"], s["refs"], s["lens"], s["pool"]
    page, most = c["page"], c["thi"]
    real, _, up, _ = _grid(s, most)
    rows, leaves = s["trees"].long(), s["leaves"].long()
    one = torch.arange(c["n"], device="cuda")
    path = up[one, leaves] & real  # the kept nodes
    base = lens[rows].long() - real.sum(-1)
    rank = torch.cumsum(path, -1) - 1
    tree, node = path.nonzero(as_tuple=True)
    src, dst = base[tree] + node, base[tree] + rank[tree, node]
    at, to = table[rows[tree], src // page].long(), table[rows[tree], dst // page].long()
    pool[:, to, :, dst % page, :] = pool[:, at, :, src % page, :]
    # the pages behind the path
    kept = base + path.sum(-1)
    j = torch.arange(table.shape[1], device="cuda")[None, :]
    old = table[rows]
    gone = (old >= 0) & (j >= -(-kept // page)[:, None])
    refs.index_add_(0, old.clamp(min=0).long().flatten(), -gone.to(torch.int32).flatten())
    table[rows] = torch.where(gone, torch.full_like(old, -1), old)
    lens[rows] = kept.to(torch.int32)
    # and room for the next tree
    have = -(-kept // page)
    need = -(-(kept + s["again"]) // page) - have
    short = need.sum() - (refs == 0).sum()
    ok = short <= 0
    order = torch.argsort((refs != 0).to(torch.uint8), stable=True)
    k = j - have[:, None]
    new = (k >= 0) & (k < need[:, None]) & ok
    got = order[((torch.cumsum(need, 0) - need)[:, None] + k).clamp(0, refs.numel() - 1)]
    refs.index_add_(0, got.flatten(), new.to(torch.int32).flatten())
    table[rows] = torch.where(new, got.to(torch.int32), table[rows])
    lens[rows] = torch.where(ok, lens[rows] + s["again"], lens[rows])
    s["status"].copy_(torch.stack([torch.zeros_like(short), short.clamp(min=0)]))
    return [table, lens, refs, s["status"], pool]


def _plain_q4(s):
    out, inner = s["case"]["out"], s["case"]["inner"]
    codes = torch.stack([s["codes"] & 15, s["codes"] >> 4], -1).view(-1, 64)
    w = (s["levels"][codes.int()] * s["scale"][:, None]).view(out, inner)
    y = torch.matmul(s["x"].float(), w.t())
    if s["bias"] is not None:
        y = y + s["bias"].float()
    return y.to(s["x"].dtype)


_run_own = dict(append=_own_append, tree=_own_tree, keep=_own_keep, q4=_own_q4)
_run_plain = dict(append=_plain_append, tree=_plain_tree, keep=_plain_keep, q4=_plain_q4)


# --- what a pass cannot do without ------------------------------------------------------------

def work(case):
    op, size = case["op"], SIZE[case["dtype"]]
    if op == "q4":
        n, out, inner = case["n"], case["out"], case["inner"]
        return {"bytes": out * inner * (0.5 + 4 / 64) + size * (n * (out + inner) + (out if case["bias"] else 0)), "flops": 2.0 * n * out * inner}
    token = case["heads"] * case["d"] * size
    if op == "append":
        return {"bytes": case["n"] * ((2.0 * case["group"] + 4.0) * token + 12) + 4.0 * case["dims"], "flops": 3.0 * case["n"] * case["heads"] * (case["group"] + 1) * case["dims"]}
    had, nodes, parents = _trees(case)
    if op == "tree":
        window, seen, read = case["window"] or 1 << 40, 0, 0
        for b, t, p in zip(had.tolist(), nodes.tolist(), parents):
            depth = _depths(p)
            seen += int((np.minimum(b, np.maximum(0, window - 1 - depth)) + np.minimum(depth + 1, window)).sum())
            read += min(b, window - 1) + t if t else 0
        n = int(nodes.sum())
        return {"bytes": 2.0 * token * (read + case["group"] * n) + 4.0 * int(_pages(had + nodes, case["page"]).sum()) + 4.0 * n,
                "flops": 4.0 * seen * case["group"] * case["heads"] * case["d"]}
    moved = 0  # tokens whose place changes
    for p, j in zip(parents, _leaves(case).tolist()):
        path = _path(p, j)
        moved += sum(a != i for i, a in enumerate(path))
    return {"bytes": 4.0 * case["layers"] * token * moved + 4.0 * int(nodes.sum()) + 16.0 * case["n"], "flops": 0.0}


def _path(parents, leaf):
    path = []
    while leaf >= 0:
        path.append(leaf)
        leaf = int(parents[leaf])
    return path[::-1]


# --- the operators in 64 bits -------------------------------------------------------------------

def exact(case, seed):
    global own
    kept, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = kept
    return dict(append=_exact_append, tree=_exact_tree, keep=_exact_keep, q4=_exact_q4)[case["op"]](case, s)


def _exact_append(case, s):
    dims, page = case["dims"], case["page"]
    with np.errstate(over="ignore"):
        turn = s["turns"].cpu().numpy().astype(np.uint64)[:, None] * s["steps"].cpu().numpy().view(np.uint64)[None, :]
    w = torch.from_numpy(np.exp(2j * math.pi * (turn.astype(np.float64) / 2.0**64))).cuda()[:, None, :]

    def turned(x):
        y = x.double().clone()
        first, second = (slice(0, dims // 2), slice(dims // 2, dims)) if case["pairs"] == "half" else (slice(0, dims, 2), slice(1, dims, 2))
        z = torch.complex(y[..., first].contiguous(), y[..., second].contiguous()) * w
        y[..., first], y[..., second] = z.real, z.imag
        return y

    out, table, k = s["pool"].double(), s["table"].cpu().numpy(), turned(s["new_k"])
    for i, (r, p) in enumerate(zip(s["rows"].tolist(), s["pos"].tolist())):
        a = int(table[r, p // page])
        out[0, a, :, p % page] = k[i]
        out[1, a, :, p % page] = s["new_v"][i].double()
    return [turned(s["q"]), out]


def _exact_tree(case, s):
    h, g, d, page = case["heads"], case["group"], case["d"], case["page"]
    _, size, parents = _trees(case)
    table, lens, starts = s["table"].cpu().numpy(), s["lens"].tolist(), s["starts"].tolist()
    out = torch.zeros(starts[-1], h * g, d, dtype=torch.float64, device="cuda")
    for i, (t, p) in enumerate(zip(size.tolist(), parents)):
        if t == 0:
            continue
        base, depth = lens[i] - t, _depths(p)
        place = np.arange(lens[i])
        logical = np.concatenate([np.arange(base), base + depth])
        up = np.zeros((t, t), dtype=bool)
        for j in range(t):
            up[j, _path(p, j)] = True
        seen = np.concatenate([np.ones((t, base), dtype=bool), up], 1)
        back = logical[None, :] - (base + depth)[:, None]
        if case["window"]:
            seen &= back > -case["window"]
        seen, back = torch.from_numpy(seen).cuda(), torch.from_numpy(back).cuda().double()
        page_of = torch.from_numpy(table[i, place // page].astype(np.int64)).cuda()
        slot = torch.from_numpy(place % page).cuda()
        for a in range(h):
            k, v = (x[page_of, a, slot, :].double() for x in s["pool"])
            for b in range(g):
                x = s["q"][starts[i]:starts[i + 1], a * g + b].double() @ k.T / math.sqrt(d)
                if case["softcap"]:
                    x = case["softcap"] * torch.tanh(x / case["softcap"])
                if case["bias"]:
                    x = x + s["slopes"][a * g + b].double() * back
                x = torch.where(seen, x, torch.full_like(x, -math.inf))
                out[starts[i]:starts[i + 1], a * g + b] = torch.softmax(x, -1) @ v
    return out


def _exact_keep(case, s):
    page, table, pool = case["page"], s["table"].cpu().numpy(), s["pool"].clone()
    _, size, parents = _trees(case)
    for i, (n, t, p, leaf) in enumerate(zip(s["lens"].tolist(), size.tolist(), parents, s["leaves"].tolist())):
        for k, j in enumerate(_path(p, leaf)):
            a, b = n - t + j, n - t + k
            pool[:, int(table[i, b // page]), :, b % page] = s["pool"][:, int(table[i, a // page]), :, a % page]
    return [None, None, None, None, pool]


def _exact_q4(case, s):
    out, inner = case["out"], case["inner"]
    y = torch.empty(case["n"], out, dtype=torch.float64, device="cuda")
    levels, x = torch.from_numpy(_levels().astype(np.float64)).cuda(), s["x"].double()
    for first in range(0, out, 2048):  # some rows of the matrix at a time
        last = min(out, first + 2048)
        codes = s["codes"][first * inner // 2:last * inner // 2].long()
        w = torch.empty(last - first, inner, dtype=torch.float64, device="cuda")
        w.view(-1)[0::2], w.view(-1)[1::2] = levels[codes % 16], levels[codes // 16]
        w.mul_(s["scale"][first * inner // 64:last * inner // 64].double().repeat_interleave(64).view(last - first, inner))
        y[:, first:last] = x @ w.T
    return y if s["bias"] is None else y + s["bias"].double()
