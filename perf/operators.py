"""The operators that write an answer with the perturbed model, as cases that can be timed and compared.

A forward-only method scores theta + eps z and theta - eps z by what the model answers. Its answers are
written token by token from a cache of keys and values in pages, which every perturbation empties:

* ``attend``  one new token of each row against its pages;
* ``write``   the new keys and values to their slots;
* ``fork``    several answers from one prompt: full pages shared, the last one copied;
* ``churn``   finished rows freed, the cache compacted, pages reserved for the next rows;
* ``sample``  the next token from its logits and a given random word.

``prepare`` makes the inputs from the seed, ``run`` makes the calls (``own``) or computes the same in
elementary torch operations, ``exact`` restates them in 64 bits, row by row.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "bf16": 2}

# heads, head size and layers of the OPT decoders, and their vocabulary
VOCAB = 50272


def listed():
    return [
        # One short answer of a small fp32 decoder (12 heads of 64): a call's latency is all.
        dict(name="attend-1x37-f32", op="attend", dtype="f32", n=1, heads=12, group=1, d=64, page=16, layout="hnd", lo=37, hi=37,
             sizes_seed=0, empty=0, window=0, softcap=0.0, bias=False),
        # A batch of ragged answers on the shape of the 6.7B decoder (32 heads of 128), a finished
        # row still in it.
        dict(name="attend-48-ragged-bf16", op="attend", dtype="bf16", n=48, heads=32, group=1, d=128, page=16, layout="hnd", lo=65, hi=2048,
             sizes_seed=1, empty=1, window=0, softcap=0.0, bias=False),
        # A few rows over very long contexts, eight query heads to a key head, scores capped.
        dict(name="attend-3-long-g8-bf16", op="attend", dtype="bf16", n=3, heads=8, group=8, d=128, page=64, layout="nhd", lo=90001, hi=131072,
             sizes_seed=2, empty=0, window=0, softcap=30.0, bias=False),
        # Many answers at once on the shape of the 13B decoder (40 heads of 128), near its 2048 positions.
        # The largest case.
        dict(name="attend-96-full-bf16", op="attend", dtype="bf16", n=96, heads=40, group=1, d=128, page=32, layout="hnd", lo=1900, hi=2048,
             sizes_seed=3, empty=0, window=0, softcap=0.0, bias=False),
        # The new token of 64 rows.
        dict(name="write-64-bf16", op="write", dtype="bf16", n=64, rows=64, lo=1, hi=500, heads=32, d=128, page=16, layout="hnd", sizes_seed=8),
        # The tokens of a batch of prompts.
        dict(name="write-8191-f32", op="write", dtype="f32", n=8191, rows=8, lo=1, hi=9, heads=12, d=64, page=16, layout="nhd", sizes_seed=9),
        # Eight answers to each of four short prompts, 12 layers.
        dict(name="fork-4x8-f32", op="fork", dtype="f32", parents=4, copies=8, lo=20, hi=90, heads=12, d=64, page=16, layout="hnd",
             layers=12, sizes_seed=4),
        # 192 answers, 24 layers of 32 heads of 64, large pages.
        dict(name="fork-24x8-bf16", op="fork", dtype="bf16", parents=24, copies=8, lo=300, hi=1500, heads=32, d=64, page=64, layout="nhd",
             layers=24, sizes_seed=5),
        # A small server's turn-over.
        dict(name="churn-2x5-bf16", op="churn", dtype="bf16", rows=5, lo=17, hi=300, heads=12, d=64, page=16, layout="hnd", layers=12, sizes_seed=6),
        # Half of 96 rows finish.
        dict(name="churn-2x48-bf16", op="churn", dtype="bf16", rows=48, lo=400, hi=2048, heads=32, d=128, page=16, layout="hnd", layers=1, sizes_seed=7),
        # One row's next token with every filter.
        dict(name="sample-1-f32", op="sample", dtype="f32", n=1, vocab=VOCAB, k=50, p=0.95, minp=0.02, banned=0.0),
        # A batch's next tokens: nucleus sampling, a tenth of the vocabulary banned.
        dict(name="sample-256-bf16", op="sample", dtype="bf16", n=256, vocab=VOCAB, k=0, p=0.9, minp=0.0, banned=0.1),
    ]


def draw(rng):
    """One more case: every operation, type and layout, sizes spread over their logarithm."""
    def log_uniform(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    op = rng.choice(["attend", "attend", "attend", "write", "fork", "churn", "sample", "sample"])
    if op == "sample":
        n = log_uniform(1, 512)
        return dict(op=op, dtype=rng.choice(["f32", "bf16"]), n=n, vocab=log_uniform(1000, min(262144, 40_000_000 // n)),
                    k=rng.choice([0, 0, log_uniform(1, 1000)]), p=rng.choice([1.0, 0.5, 0.9, 0.97]), minp=rng.choice([0.0, 0.0, 0.05]),
                    banned=rng.choice([0.0, 0.3]))
    case = dict(op=op, dtype=rng.choice(["f32", "bf16", "bf16"]), page=rng.choice([16, 16, 32, 48, 64, 128]), layout=rng.choice(["hnd", "nhd"]),
                d=rng.choice([64, 64, 80, 96, 128, 128, 256]), sizes_seed=rng.randrange(1 << 30))
    if op == "attend":
        case.update(n=log_uniform(1, 400), group=rng.choice([1, 1, 2, 4, 5, 8, 16]))
        case["heads"] = min(log_uniform(1, 40), max(1, 128 // case["group"]))
        most = int(1.2e9 / (SIZE[case["dtype"]] * case["n"] * case["heads"] * case["d"]))  # tokens of a row, at most
        case["hi"] = log_uniform(1, max(1, min(131072, most)))
        case["lo"] = rng.choice([1, max(1, case["hi"] // 2), case["hi"]])
        case.update(empty=rng.choice([0, 1]) if case["n"] > 1 else 0, window=rng.choice([0, 0, log_uniform(1, 4096)]),
                    softcap=rng.choice([0.0, 0.0, 30.0]), bias=rng.random() < 0.3)
    elif op == "write":
        case.update(n=log_uniform(1, 8192), heads=log_uniform(1, 40), lo=1, hi=log_uniform(1, 1000))
        case["rows"] = min(case["n"], log_uniform(1, 256))
    elif op == "fork":
        case.update(parents=log_uniform(1, 32), copies=log_uniform(1, 16), heads=log_uniform(1, 32), layers=log_uniform(1, 24))
        token = 2 * case["layers"] * case["heads"] * case["d"] * SIZE[case["dtype"]]
        rows = case["parents"] * (1 + 2 * case["copies"])  # the prompts, and two last pages for each answer
        case["hi"] = log_uniform(1, max(2, min(4096, int(2e9 / token / case["parents"]) - rows * case["page"] // case["parents"])))
        case["lo"] = max(1, case["hi"] // 4)
    else:
        case.update(rows=log_uniform(1, 64), heads=log_uniform(1, 32), layers=log_uniform(1, 8))
        token = 2 * case["layers"] * case["heads"] * case["d"] * SIZE[case["dtype"]]
        case["hi"] = log_uniform(1, max(2, min(4096, int(2e9 / token / (2 * case["rows"])))))
        case["lo"] = max(1, case["hi"] // 4)
    return case


# --- shapes -------------------------------------------------------------------------------

def _lens(case, n):
    """Lengths of n rows, spread over their logarithm: the first the longest, `empty` of the others 0."""
    g = np.random.default_rng(case["sizes_seed"])
    v = np.exp(g.uniform(math.log(case["lo"]), math.log(case["hi"] + 1), size=n)).astype(np.int64).clip(case["lo"], case["hi"])
    v[0] = case["hi"]
    if case.get("empty"):
        v[n // 2] = 0
    return v


def _pages(lens, page):
    return -(-lens // page)


def _pool(case, n_pages, layers, seed):
    """Keys and values [2 layers, pages, heads, tokens, d], N(0, 1), in memory by heads or by tokens."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    h, p, d = case["heads"], case["page"], case["d"]
    shape = (2 * layers, n_pages, h, p, d) if case["layout"] == "hnd" else (2 * layers, n_pages, p, h, d)
    x = torch.empty(shape, dtype=DTYPES[case["dtype"]], device="cuda").normal_(generator=g)
    return x if case["layout"] == "hnd" else x.transpose(2, 3)


def _table(lens, case, n_pages, row_pages, g, among=None):
    """Page ids of rows of these lengths in a random order of the first `among` pages, and their references."""
    table = np.full((len(lens), row_pages), -1, dtype=np.int32)
    need = _pages(lens, case["page"])
    ids = g.permutation(int(need.sum()) if among is None else among)[:int(need.sum())].astype(np.int32)
    table[np.arange(row_pages)[None, :] < need[:, None]] = ids
    refs = np.zeros(n_pages, dtype=np.int32)
    refs[ids] = 1
    return table, refs


def _cuda(a, dtype=None):
    return torch.from_numpy(np.ascontiguousarray(a)).to("cuda", dtype=dtype)


def prepare(case, seed):
    g = np.random.default_rng([seed, 3])
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed + 1)
    s = dict(case=case)
    op = case["op"]
    if op == "sample":
        n, v = case["n"], case["vocab"]
        # a vocabulary's logits: a few likely tokens, a long tail
        rank = torch.rand(n, v, device="cuda", generator=gen)
        x = 1.5 * torch.randn(n, v, device="cuda", generator=gen) - 1.1 * torch.log1p(v * rank) + 10
        if case["banned"]:
            x[torch.rand(n, v, device="cuda", generator=gen) < case["banned"]] = -math.inf
        s["logits"] = x.to(DTYPES[case["dtype"]])
        s["words"] = _cuda(g.integers(0, 1 << 32, size=n, dtype=np.uint64).astype(np.uint32).view(np.int32))
        t = g.uniform(0.6, 1.4, size=n)
        t[np.arange(n) % 16 == 7] = 0.0  # greedy rows among the others
        s["temperature"] = _cuda(t, torch.float32)
        s["top_k"] = _cuda(np.full(n, case["k"]) + (g.integers(0, 20, size=n) if case["k"] else 0), torch.int32)
        s["top_p"] = _cuda(np.full(n, case["p"]), torch.float32)
        s["min_p"] = _cuda(np.full(n, case["minp"]), torch.float32)
        return s
    page, layers = case["page"], 1
    if op == "attend":
        lens = _lens(case, case["n"])
        need = int(_pages(lens, page).sum())
        row_pages, n_pages = int(_pages(lens, page).max()), need + 3
        table, refs = _table(lens, case, n_pages, row_pages, g, among=n_pages)
        n, h, d = case["n"], case["heads"], case["d"]
        # the queries as the projection leaves them, beside the row's new keys and values
        qkv = torch.randn(n, (case["group"] + 2) * h * d, device="cuda", generator=gen)
        qkv[:, :case["group"] * h * d] *= 2.5  # some tokens stand out
        s["q"] = qkv.to(DTYPES[case["dtype"]])[:, :case["group"] * h * d].view(n, case["group"] * h, d)
        s["pos"] = _cuda(lens - 1, torch.int32)
        s["rows"] = torch.arange(n, dtype=torch.int32, device="cuda")
        s["slopes"] = (2.0 ** -torch.linspace(1, 8, case["group"] * h, device="cuda")).float() if case["bias"] else None
    elif op == "write":
        # each row's share of the n tokens, after the tokens that it has
        n, h, d = case["n"], case["heads"], case["d"]
        had, new = _lens(case, case["rows"]), np.diff(np.arange(case["rows"] + 1) * n // case["rows"])
        lens = had + new
        row_pages, n_pages = int(_pages(lens, page).max()), int(_pages(lens, page).sum()) + 3
        table, refs = _table(lens, case, n_pages, row_pages, g, among=n_pages)
        rows = np.repeat(np.arange(case["rows"]), new)
        s["rows"] = _cuda(rows, torch.int32)
        s["pos"] = _cuda(had[rows] + np.arange(n) - (np.cumsum(new) - new)[rows], torch.int32)
        kv = torch.randn(n, 2 * h * d, device="cuda", generator=gen).to(DTYPES[case["dtype"]])
        s["new_k"], s["new_v"] = kv[:, :h * d].view(n, h, d), kv[:, h * d:].view(n, h, d)
    elif op == "fork":
        lens, parents, children = _fork_rows(case)
        need, partial = int(_pages(lens, page).sum()), int((lens[parents] % page > 0).sum())
        row_pages, n_pages = int(_pages(lens, page).max()), need + 2 * partial + 1
        among = np.zeros(len(parents), dtype=np.int64)
        table, refs = _table(np.concatenate([lens, among]), case, n_pages, row_pages, g, among=n_pages)
        lens = np.concatenate([lens, among])
        layers = case["layers"]
        s["parents"], s["children"] = _cuda(parents, torch.int32), _cuda(children, torch.int32)
    else:
        lens = _lens(case, 2 * case["rows"])
        need = int(_pages(lens, page).sum())
        row_pages, n_pages = int(_pages(lens, page).max()), need + 2
        table, refs = _table(lens, case, n_pages, row_pages, g)
        layers = case["layers"]
        half = [np.arange(i, 2 * case["rows"], 2) for i in (0, 1)]
        s["halves"] = [(_cuda(h, torch.int32), _cuda(lens[h], torch.int32)) for h in half]
        s["turn"] = 0
    s["pool"] = _pool(case, n_pages, layers, seed)
    s["table"], s["refs"], s["lens"] = _cuda(table), _cuda(refs), _cuda(lens, torch.int32)
    s["status"] = torch.zeros(1, dtype=torch.int32, device="cuda")
    if own:
        import paper_2306_10015_gb300 as jb
        pages = jb.PageTable(s["table"], s["lens"], s["refs"], page)
        s["cache"] = jb.KVCache(pages, list(s["pool"][:layers]), list(s["pool"][layers:]))
    return s


def _fork_rows(case):
    lens = _lens(case, case["parents"])
    n = case["parents"] * case["copies"]
    return lens, np.arange(n) // case["copies"], case["parents"] + np.arange(n)


# --- one pass -------------------------------------------------------------------------------

def run(state):
    op = state["case"]["op"]
    return (_run_own if own else _run_plain)[op](state)


def _own_attend(s):
    import paper_2306_10015_gb300 as jb
    c = s["case"]
    return jb.jb_attend(s["cache"], 0, s["q"], s["rows"], s["pos"], softcap=c["softcap"], window=c["window"], slopes=s["slopes"])


def _own_write(s):
    import paper_2306_10015_gb300 as jb
    jb.jb_cache_write(s["cache"], 0, s["new_k"], s["new_v"], s["rows"], s["pos"])
    return s["pool"]


def _own_fork(s):
    import paper_2306_10015_gb300 as jb
    jb.jb_cache_fork(s["cache"], s["parents"], s["children"], status=s["status"])
    return [s["table"], s["lens"], s["refs"], s["status"], s["pool"]]


def _own_churn(s):
    import paper_2306_10015_gb300 as jb
    rows, tokens = s["halves"][s["turn"]]
    s["turn"] ^= 1
    jb.jb_cache_free(s["cache"], rows)
    jb.jb_cache_compact(s["cache"])
    jb.jb_cache_reserve(s["cache"], rows, tokens, status=s["status"])
    return [s["table"], s["lens"], s["refs"], s["status"], s["pool"]]


def _own_sample(s):
    import paper_2306_10015_gb300 as jb
    return list(jb.jb_sample(s["logits"], s["words"], temperature=s["temperature"], top_k=s["top_k"], top_p=s["top_p"], min_p=s["min_p"]))


def _plain_attend(s):
    c = s["case"]
    n, h, g, d, page = c["n"], c["heads"], c["group"], c["d"], c["page"]
    table = s["table"][s["rows"].long()].long().clamp(min=0)
    span = table.shape[1] * page
    k, v = (x[table].permute(0, 2, 1, 3, 4).reshape(n, h, span, d).float() for x in s["pool"])
    x = torch.matmul(s["q"].float().reshape(n, h, g, d), k.transpose(-1, -2)) * (1.0 / math.sqrt(d))
    if c["softcap"]:
        x = c["softcap"] * torch.tanh(x / c["softcap"])
    back = torch.arange(span, device="cuda")[None, :] - s["pos"].long()[:, None]
    if c["bias"]:
        x = x + s["slopes"].view(1, h, g, 1) * back[:, None, None, :].float()
    seen = back <= 0
    if c["window"]:
        seen = seen & (back > -c["window"])
    seen = seen[:, None, None, :]
    top = torch.where(seen, x, torch.full_like(x, -3e38)).amax(-1, keepdim=True)
    e = torch.where(seen, torch.exp(x - top), torch.zeros_like(x))
    out = torch.matmul(e, v) / e.sum(-1, keepdim=True).clamp(min=1e-30)
    return out.reshape(n, h * g, d).to(s["q"].dtype)


def _plain_write(s):
    pos, page = s["pos"].long(), s["case"]["page"]
    at = s["table"][s["rows"].long(), pos // page].long()
    s["pool"][0][at, :, pos % page, :] = s["new_k"]
    s["pool"][1][at, :, pos % page, :] = s["new_v"]
    return s["pool"]


def _plain_fork(s):
    page, table, refs, lens = s["case"]["page"], s["table"], s["refs"], s["lens"]
    parents, children = s["parents"].long(), s["children"].long()
    old, rows, n = table[children], table[parents], lens[parents].long()
    need = (n % page > 0) & (parents != children)
    free = refs == 0
    short = need.sum() - free.sum()
    ok = short <= 0
    order = torch.argsort((~free).to(torch.uint8), stable=True)
    fresh = order[(torch.cumsum(need, 0) - 1).clamp(0, refs.numel() - 1)]
    at = (n // page).clamp(max=table.shape[1] - 1)
    one = torch.arange(len(parents), device="cuda")
    last = rows[one, at].long()
    rows[one, at] = torch.where(need, fresh.to(torch.int32), rows[one, at])
    move = ((parents != children) & ok)[:, None]
    refs.index_add_(0, old.clamp(min=0).long().flatten(), -((old >= 0) & move).to(torch.int32).flatten())
    refs.index_add_(0, rows.clamp(min=0).long().flatten(), ((rows >= 0) & move).to(torch.int32).flatten())
    table[children] = torch.where(move, rows, old)
    lens[children] = torch.where(move[:, 0], n.to(torch.int32), lens[children])
    s["status"].copy_(short.clamp(min=0).view(1))
    which = (need & ok).nonzero().flatten()
    dst, src = fresh[which], last[which]
    seen = torch.arange(page, device="cuda")[None, :] < (n % page)[which][:, None]
    pool = s["pool"]
    pool[:, dst] = torch.where(seen[None, :, None, :, None], pool[:, src], pool[:, dst])
    return [table, lens, refs, s["status"], pool]


def _plain_churn(s):
    page, table, refs, lens, pool = s["case"]["page"], s["table"], s["refs"], s["lens"], s["pool"]
    rows, tokens = s["halves"][s["turn"]]
    rows, tokens = rows.long(), tokens.long()
    s["turn"] ^= 1
    # free
    old = table[rows]
    refs.index_add_(0, old.clamp(min=0).long().flatten(), -(old >= 0).to(torch.int32).flatten())
    table[rows] = -1
    lens[rows] = 0
    # compact
    ids = torch.arange(refs.numel(), device="cuda")
    live = refs > 0
    n_live = live.sum()
    src, dst = (live & (ids >= n_live)).nonzero().flatten(), (~live & (ids < n_live)).nonzero().flatten()
    moved = ids.clone()
    moved[src] = dst
    pool[:, dst] = pool[:, src]
    refs[dst] = refs[src]
    refs[src] = 0
    table.copy_(torch.where(table >= 0, moved[table.clamp(min=0).long()].to(torch.int32), table))
    # reserve
    have = -(-lens[rows].long() // page)
    need = -(-(lens[rows] + tokens) // page) - have
    short = need.sum() - (refs == 0).sum()
    ok = short <= 0
    order = torch.argsort((refs != 0).to(torch.uint8), stable=True)
    j = torch.arange(table.shape[1], device="cuda")[None, :] - have[:, None]
    new = (j >= 0) & (j < need[:, None]) & ok
    got = order[((torch.cumsum(need, 0) - need)[:, None] + j).clamp(0, refs.numel() - 1)]
    refs.index_add_(0, got.flatten(), new.to(torch.int32).flatten())
    table[rows] = torch.where(new, got.to(torch.int32), table[rows])
    lens[rows] = torch.where(ok, lens[rows] + tokens.to(torch.int32), lens[rows])
    s["status"].copy_(short.clamp(min=0).view(1))
    return [table, lens, refs, s["status"], pool]


def _plain_sample(s):
    x = s["logits"].float()
    x = torch.where(torch.isnan(x), torch.full_like(x, -math.inf), x)
    top = x.amax(-1, keepdim=True)
    temperature = s["temperature"][:, None]
    greedy = ~(temperature >= 2.0**-64)
    y = (x - top) * (1.0 / torch.where(greedy, torch.ones_like(temperature), temperature))
    y = torch.where(x == top, torch.zeros_like(y), y)
    w = torch.round(torch.exp(y) * 2.0**30).long()
    _, order = torch.sort(x, dim=-1, descending=True, stable=True)
    ws = torch.gather(w, 1, order)
    rank = torch.arange(x.shape[1], device="cuda")[None, :]
    k = s["top_k"].long()[:, None]
    k = torch.where(greedy, torch.ones_like(k), torch.where(k <= 0, torch.full_like(k, x.shape[1]), k))
    ws = torch.where(rank < k, ws, torch.zeros_like(ws))
    running = torch.cumsum(ws, -1)
    p = s["top_p"].double()[:, None]
    mass = torch.ceil(torch.where(p < 1, p, torch.ones_like(p)) * running[:, -1:].double()).long().clamp(min=1)
    cut = torch.ceil(s["min_p"].double().clamp(0, 1) * 2.0**30).long()[:, None]
    ws = torch.where((running - ws < mass) & (ws >= cut), ws, torch.zeros_like(ws))
    kept = torch.zeros_like(ws).scatter_(1, order, ws)
    running = torch.cumsum(kept, -1)
    total = running[:, -1:]
    word = s["words"].long()[:, None] & 0xFFFFFFFF
    # floor(word total / 2^32) with total < 2^48, by halves of the word
    aim = ((word >> 16) * total + (((word & 0xFFFF) * total) >> 16)) >> 16
    token = (running <= aim).sum(-1, keepdim=True).clamp(max=x.shape[1] - 1)
    logprob = torch.gather(y, 1, token) - torch.log(total.float() * 2.0**-30)
    none = torch.isinf(top) & (top < 0)
    token = torch.where(none, torch.full_like(token, -1), token)
    logprob = torch.where(none, torch.full_like(logprob, -math.inf), logprob)
    return [token[:, 0].to(torch.int32), logprob[:, 0]]


_run_own = dict(attend=_own_attend, write=_own_write, fork=_own_fork, churn=_own_churn, sample=_own_sample)
_run_plain = dict(attend=_plain_attend, write=_plain_write, fork=_plain_fork, churn=_plain_churn, sample=_plain_sample)


# --- what a pass cannot do without ------------------------------------------------------------

def work(case):
    op, size = case["op"], SIZE[case["dtype"]]
    if op == "sample":
        return {"bytes": case["n"] * (case["vocab"] * size + 28.0), "flops": 2.0 * case["n"] * case["vocab"]}
    token = case["heads"] * case["d"] * size
    page = case["page"]
    if op == "attend":
        lens = _lens(case, case["n"])
        seen = int(np.minimum(lens, case["window"] or lens).sum())
        return {"bytes": 2.0 * token * (seen + case["group"] * case["n"]) + 4.0 * int(_pages(lens, page).sum()),
                "flops": 4.0 * seen * case["group"] * case["heads"] * case["d"]}
    if op == "write":
        return {"bytes": case["n"] * (4.0 * token + 12), "flops": 0.0}
    if op == "fork":
        lens, parents, _ = _fork_rows(case)
        rows = 4.0 * int(_pages(lens, page)[parents].sum())  # entries read, written, counted
        return {"bytes": 4.0 * case["layers"] * token * int((lens[parents] % page).sum()) + 3 * rows, "flops": 0.0}
    # churn: one half's pages are below the other's from the second pass on, and are freed: as many
    # pages move down as both halves have
    lens = _lens(case, 2 * case["rows"])
    a, b = (int(_pages(lens[i::2], page).sum()) for i in (0, 1))
    return {"bytes": 4.0 * case["layers"] * token * page * min(a, b) + 12.0 * (a + b), "flops": 0.0}


# --- the operators in 64 bits -------------------------------------------------------------------

def exact(case, seed):
    global own
    kept, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = kept
    return dict(attend=_exact_attend, write=_exact_write, fork=_exact_fork, churn=_exact_churn, sample=_exact_sample)[case["op"]](case, s)


def _exact_attend(case, s):
    h, g, d = case["heads"], case["group"], case["d"]
    out = torch.zeros(case["n"], h * g, d, dtype=torch.float64, device="cuda")
    table, pos = s["table"].cpu().numpy(), s["pos"].cpu().numpy()
    for i, last in enumerate(pos.tolist()):
        if last < 0:
            continue
        first = max(0, last - case["window"] + 1) if case["window"] else 0
        at = np.arange(first, last + 1)
        page = torch.from_numpy(table[i, at // case["page"]].astype(np.int64)).cuda()
        slot = torch.from_numpy(at % case["page"]).cuda()
        k, v = (x[page, :, slot, :].double().transpose(0, 1) for x in s["pool"])  # [heads, tokens, d]
        x = torch.einsum("hgd,htd->hgt", s["q"][i].double().view(h, g, d), k) / math.sqrt(d)
        if case["softcap"]:
            x = case["softcap"] * torch.tanh(x / case["softcap"])
        if case["bias"]:
            x = x + s["slopes"].double().view(h, g, 1) * torch.from_numpy((at - last).astype(np.float64)).cuda()
        out[i] = torch.einsum("hgt,htd->hgd", torch.softmax(x, -1), v).reshape(h * g, d)
    return out


def _exact_write(case, s):
    out = s["pool"].clone()
    table = s["table"].cpu().numpy()
    for i, (r, p) in enumerate(zip(s["rows"].tolist(), s["pos"].tolist())):
        a = int(table[r, p // case["page"]])
        out[0, a, :, p % case["page"]] = s["new_k"][i]
        out[1, a, :, p % case["page"]] = s["new_v"][i]
    return out


def _exact_fork(case, s):
    table, lens, refs, page = s["table"].cpu().numpy(), s["lens"].cpu().numpy(), s["refs"].cpu().numpy(), case["page"]
    free, pool = [int(p) for p in np.flatnonzero(refs == 0)], s["pool"].clone()
    for a, b in zip(s["parents"].tolist(), s["children"].tolist()):
        if lens[a] % page:  # the children's rows are empty at first: nothing to release
            pool[:, free.pop(0), :, :lens[a] % page] = s["pool"][:, int(table[a, lens[a] // page]), :, :lens[a] % page]
    return [None, None, None, None, pool]


def _exact_churn(case, s):
    refs, table = s["refs"].cpu().numpy(), s["table"].cpu().numpy()
    rows = s["halves"][0][0].cpu().numpy()
    gone = table[rows]
    refs[gone[gone >= 0]] = 0
    n_live, pool = int((refs > 0).sum()), s["pool"].clone()
    holes = iter(np.flatnonzero(refs == 0).tolist())
    for p in np.flatnonzero(refs > 0).tolist():
        if p >= n_live:
            pool[:, next(holes)] = s["pool"][:, p]
    return [None, None, None, None, pool]


def _exact_sample(case, s):
    logprob = []
    for i in range(case["n"]):
        x, t = s["logits"][i].double(), float(s["temperature"][i])
        w = torch.round(torch.exp((x - x.max()) / (t or 1.0)) * 2.0**30)
        order = torch.sort(x, descending=True, stable=True)[1]
        k = 1 if t == 0 else int(s["top_k"][i]) or case["vocab"]
        order, mass = order[:k], w[order[:k]].cumsum(0)
        need = max(1.0, math.ceil(min(1.0, float(s["top_p"][i])) * float(mass[-1])))
        keep = order[(mass - w[order] < need) & (w[order] >= math.ceil(float(s["min_p"][i]) * 2**30))]
        z = torch.zeros_like(w)
        z[keep] = w[keep]
        total = int(z.sum())
        aim = ((int(s["words"][i]) & 0xFFFFFFFF) * total) >> 32
        token = int((z.cumsum(0) <= aim).sum())
        logprob.append(float(x[token] - x.max()) / (t or 1.0) - math.log(total / 2.0**30))
    return [None, torch.tensor(logprob, dtype=torch.float64)]
