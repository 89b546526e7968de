"""jb_attend_tree against the definition in 64 bits, where it can go wrong: trees from one node to 256, chains and bushes,
rows around pages and tiles, heads that share keys, head sizes between the kernels', windows by depth, what unseen places
hold, invalid trees and parents, strides, streams, graphs.

Tolerances as in test_gpu_attend.py, with A = sum_t p_t |v_t| and S = max_t scale sum_e |q_e k_e| of a node's query: scores
off by (d + 16) 2^-23 S' enter twice, exponentials 2^-21, sums of T terms T 2^-23, weights of bf16 products 2^-16, and the
result's own rounding, half a step of it: 2^-8 for bf16 (2^-9 and as much again for the tie).
"""
import math

import pytest
import torch

import paper_2306_10015_gb300 as jb
from test_gpu_attend import DT, i32, make, query

pytestmark = pytest.mark.gpu


def chain(n):
    return [j - 1 for j in range(n)]


def bush(n, seed=0, roots=1):
    g = torch.Generator().manual_seed(seed + n)
    return [-1 if j < roots else int(torch.randint(max(-1, j - 5), j, (1,), generator=g)) for j in range(n)]


def wide(n):
    return [-1 if j == 0 else (j - 1) // 4 for j in range(n)]


def draft(rows, parents):
    starts = [0]
    for p in parents:
        starts.append(starts[-1] + len(p))
    return jb.DraftTrees(i32(rows), i32(starts), i32([x for p in parents for x in p]))


def path_to(parents, j):
    """j and its ancestors, None if the chain is not valid."""
    path = []
    while j != -1:
        path.append(j)
        if not -1 <= parents[j] < j:
            return None
        j = parents[j]
    return path[::-1]


def reference(cache, layer, q, rows, parents, scale=None, softcap=0.0, window=0, slopes=None):
    """(result, tolerance) of every element in 64 bits."""
    n, qh, d = q.shape
    g = qh // cache.heads
    scale = d ** -0.5 if scale is None else scale
    page = cache.pages.page_tokens
    out = torch.zeros(n, qh, d, dtype=torch.float64, device="cuda")
    tol = torch.full_like(out, 1e-38)
    table, lens = cache.pages.table.cpu(), cache.pages.lens.tolist()
    first = 0
    for r, tree in zip(rows, parents):
        base = lens[r] - len(tree) if 0 <= r < len(lens) else -1
        for j in range(len(tree)):
            path = path_to(tree, j)
            if path is None or base < 0 or len(tree) > 256:
                continue
            where = list(range(base)) + [base + k for k in range(len(path))]     # logical positions
            place = torch.tensor(list(range(base)) + [base + k for k in path])
            here = base + len(path) - 1
            keep = torch.tensor([not window or w > here - window for w in where])
            place, back = place[keep], torch.tensor(where)[keep].cuda() - here
            ids = table[r, place // page].long()
            ok = ids >= 0
            place, back, ids = place[ok], back[ok.cuda()], ids[ok]
            if len(place) == 0:
                continue
            k = cache.keys[layer][ids.cuda(), :, (place % page).cuda()].double().repeat_interleave(g, 1)
            v = cache.values[layer][ids.cuda(), :, (place % page).cuda()].double().repeat_interleave(g, 1)
            prod = q[first + j].double()[None] * k * scale
            x, size = prod.sum(-1), prod.abs().sum(-1).amax(0)
            if softcap:
                x = softcap * torch.tanh(x / softcap)
                size = size + softcap
            if slopes is not None:
                x = x + slopes.double()[None] * back.double()[:, None]
                size = size + slopes.double() * float(-back.min())
            p = torch.softmax(x, 0)
            out[first + j] = torch.einsum("th,thd->hd", p, v)
            a = torch.einsum("th,thd->hd", p, v.abs())
            rel = 2 * (2 * (d + 16) * 2.0**-23 * size + 2.0**-21) + len(place) * 2.0**-23
            if q.dtype == torch.bfloat16:
                rel = rel + 2.0**-16
            tol[first + j] += a * rel[:, None] + (2.0**-8 * out[first + j].abs() if q.dtype == torch.bfloat16 else 0)
        first += len(tree)
    return out, tol


def check(cache, layer, q, rows, parents, **kw):
    got = jb.jb_attend_tree(cache, layer, q, draft(rows, parents), **kw)
    want, tol = reference(cache, layer, q, rows, parents, **{k: v for k, v in kw.items() if k not in ("out", "stream", "workspace")})
    torch.cuda.synchronize()
    assert torch.isfinite(got).all()
    err = (got.double() - want).abs()
    worst = (err / tol).amax() if err.numel() else 0.0
    assert (err <= tol).all(), f"worst error over tolerance {worst:.3g}"
    return got


def case(dtype, tokens, trees, heads, group, d, page, layout="hnd", **kw):
    """A cache whose row i has tokens[i] tokens and then tree i; queries."""
    cache = make(dtype, [t + len(p) for t, p in zip(tokens, trees)], heads, d, page, layout, **kw)
    return cache, query(sum(len(p) for p in trees), heads * group, d, dtype)


TOKENS = [0, 1, 15, 16, 17, 33, 63, 64, 100, 127, 128, 129, 250, 0, 511]
SIZES = [1, 2, 3, 16, 5, 31, 32, 33, 7, 64, 1, 65, 6, 40, 9]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("page,layout", [(16, "hnd"), (48, "nhd"), (128, "hnd"), (64, "nhd")])
def test_lengths_around_pages_and_tiles(dtype, page, layout):
    trees = [bush(n, i) for i, n in enumerate(SIZES)]
    cache, q = case(dtype, TOKENS, trees, 3, 1, 64, page, layout)
    check(cache, 0, q, range(len(trees)), trees)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("d", [8, 16, 40, 64, 72, 80, 96, 120, 128, 136, 192, 256])
@pytest.mark.parametrize("group", [1, 3])
def test_head_sizes(dtype, d, group):
    trees = [bush(5), chain(30), wide(12)]
    cache, q = case(dtype, [3, 200, 61], trees, 2, group, d, 32)
    check(cache, 0, q, range(3), trees)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("heads,group", [(1, 1), (4, 2), (1, 5), (2, 7), (1, 8), (3, 9), (1, 16), (1, 27), (1, 64)])
@pytest.mark.parametrize("layout", ["hnd", "nhd"])
def test_shared_heads(dtype, heads, group, layout):
    trees = [bush(6), wide(19), chain(1)]
    cache, q = case(dtype, [2, 150, 77], trees, heads, group, 128, 16, layout)
    check(cache, 0, q, range(3), trees)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("tree", [chain(256), bush(256, 3, 2), wide(255), [-1] * 200], ids=["chain", "bush", "wide", "flat"])
@pytest.mark.parametrize("heads,group,d", [(2, 1, 64), (1, 3, 128)])
def test_large_trees(dtype, tree, heads, group, d):
    trees = [tree, chain(3)]
    cache, q = case(dtype, [37, 300], trees, heads, group, d, 16)
    check(cache, 0, q, range(2), trees)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("window", [0, 1, 2, 5, 16, 31, 64, 5000])
@pytest.mark.parametrize("softcap,bias", [(0.0, False), (20.0, False), (0.0, True), (5.0, True)])
def test_windows_caps_and_biases(dtype, window, softcap, bias):
    trees = [bush(9), chain(40), wide(30), chain(2)]
    cache, _ = case(dtype, [1, 140, 20, 0], trees, 2, 3, 64, 16)
    q = query(sum(map(len, trees)), 6, 64, dtype, std=4.0)
    slopes = 2.0 ** -torch.arange(1, 7, device="cuda").float() if bias else None
    check(cache, 0, q, range(4), trees, window=window, softcap=softcap, slopes=slopes)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_long_windows_reach_into_the_row(dtype):
    trees = [chain(100), bush(33)]
    cache, q = case(dtype, [700, 400], trees, 2, 1, 64, 16)
    for window in (90, 128, 129, 200, 650):
        check(cache, 0, q, range(2), trees, window=window)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("heads,tokens", [(1, [50_001]), (2, [30_000, 1, 16_384])])
def test_long_rows_are_split_and_joined(dtype, heads, tokens):
    trees = [bush(9), chain(4), wide(7)][:len(tokens)]
    cache, q = case(dtype, tokens, trees, heads, 2, 128, 64, std=0.5)
    check(cache, 0, q, range(len(tokens)), trees)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_a_chain_is_what_single_queries_give(dtype):
    """Two roundings of the same sums: each within its own tolerance."""
    trees = [chain(70)]
    cache, q = case(dtype, [55], trees, 2, 2, 64, 16)
    got = check(cache, 0, q, [0], trees)
    want, tol = reference(cache, 0, q, [0], trees)
    one = jb.jb_attend(cache, 0, q, i32([0] * 70), i32(range(55, 125)))
    assert ((one.double() - got.double()).abs() <= 2 * tol).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("what", ["keys", "values", "both"])
def test_what_is_not_seen_has_no_effect(dtype, bad, what):
    """Keys and values of a node that are not finite reach its descendants alone; those of places behind the row, and of
    pages before a window, nobody (make() fills what no token has with NaN)."""
    tree = [-1, 0, 0, 1, 2, 3, 2]                      # below node 2: 4 and 6
    cache, q = case(dtype, [40], [tree], 2, 2, 64, 16)
    page, slot = int(cache.pages.table[0, 42 // 16]), 42 % 16
    clean = jb.jb_attend_tree(cache, 0, q, draft([0], [tree]))
    for x in {"keys": cache.keys, "values": cache.values, "both": cache.keys + cache.values}[what]:
        x[page, :, slot, ::3] = bad
    got = jb.jb_attend_tree(cache, 0, q, draft([0], [tree]))
    away = [0, 1, 3, 5]
    assert torch.equal(got[away], clean[away]) and torch.isfinite(got[away]).all()
    if what != "keys":
        assert not torch.isfinite(got[[2, 4, 6]]).all()
    for window in (1, 3):
        cache2, q2 = case(dtype, [90], [chain(2)], 1, 1, 64, 16)
        cache2.values[0][cache2.pages.table[0, :5].long()] = bad
        cache2.keys[0][cache2.pages.table[0, :5].long()] = bad
        assert torch.isfinite(jb.jb_attend_tree(cache2, 0, q2, draft([0], [chain(2)]), window=window)).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_values_that_are_not_finite_below_a_window(dtype):
    """A position that the deeper nodes' windows leave behind, in the tile where the windows begin."""
    trees = [chain(20)]
    cache, q = case(dtype, [200], trees, 2, 1, 64, 16)
    clean = jb.jb_attend_tree(cache, 0, q, draft([0], trees), window=32)
    at = 200 - 32 + 1 + 4                              # seen by nodes 0 to 4
    cache.values[0][int(cache.pages.table[0, at // 16]), :, at % 16] = math.inf
    got = jb.jb_attend_tree(cache, 0, q, draft([0], trees), window=32)
    assert torch.equal(got[5:], clean[5:])
    assert not torch.isfinite(got[:5]).any()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_missing_pages_are_not_seen(dtype):
    trees = [bush(40), chain(20)]
    cache, q = case(dtype, [160, 33], trees, 2, 1, 64, 16)
    cache.pages.table[0, 3] = -1
    cache.pages.table[0, 7:9] = -1
    cache.pages.table[0, 11] = -1                      # some nodes' own
    cache.pages.table[1, 0] = -1
    check(cache, 0, q, range(2), trees, scale=0.3)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_rows_that_see_nothing_at_all(dtype):
    trees = [chain(3)]
    cache, q = case(dtype, [20], trees, 2, 1, 64, 16)
    cache.pages.table[0] = -1
    out = torch.full_like(q, math.nan)
    assert (check(cache, 0, q, [0], trees, out=out) == 0).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_invalid_parents_and_trees(dtype):
    """Chains through an index not below their own, or below -1, give zeros; so do trees whose row is not there or too
    short, and trees of more than 256 nodes. The others are not touched by it."""
    trees = [[-1, 0, 2, 1, 2, 4, 0], chain(4), [-2, 0, -1, 2, 7], chain(257), chain(9), [-1, 0], chain(5)]
    rows = [0, 5, 1, 2, 3, -1, 4]
    cache = make(dtype, [30, 25, 300, 4, 50], 2, 64, 16)
    q = query(sum(map(len, trees)), 4, 64, dtype)
    out = torch.full_like(q, math.nan)
    got = check(cache, 0, q, rows, trees, out=out)
    starts = [0, 7, 11, 16, 273, 282, 284, 289]
    zero = [2, 4, 5] + list(range(7, 11)) + [11, 12, 15] + list(range(16, 273)) + list(range(273, 284))
    assert (got[zero] == 0).all() and starts[-1] == got.shape[0]
    assert (got[[0, 1, 3, 6, 13, 14, 284, 288]] != 0).any(-1).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_queries_of_no_tree_are_left(dtype):
    cache = make(dtype, [30, 25], 2, 64, 16)
    q = query(20, 2, 64, dtype)
    trees = jb.DraftTrees(i32([1, 0]), i32([4, 9, 15]), i32([7, 7, 7, 7] + chain(5) + bush(6) + [9] * 5))
    out = torch.full_like(q, 3.0)
    jb.jb_attend_tree(cache, 0, q, trees, out=out)
    assert (out[:4] == 3).all() and (out[15:] == 3).all()
    want = jb.jb_attend_tree(cache, 0, q[4:15], draft([1, 0], [chain(5), bush(6)]))
    assert torch.equal(out[4:15], want)
    none = jb.DraftTrees(i32([0]), i32([15, 15]), i32([0] * 20))
    jb.jb_attend_tree(cache, 0, q, none, out=out)
    assert torch.equal(out[4:15], want)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_lists_that_do_not_ascend_stay_inside(dtype):
    """Bounds that make no tree: nothing outside the outputs is touched, nothing else is said."""
    cache = make(dtype, [40, 40, 40, 40], 2, 64, 16)
    q = query(12, 2, 64, dtype)
    guard = torch.full((14, 2, 64), 5.0, dtype=DT[dtype], device="cuda")
    for starts in ([0, 9, 4, 12, 30], [-3, 2, 1 << 30, -(1 << 31), (1 << 31) - 1], [12, 12, 12, 12, 13]):
        jb.jb_attend_tree(cache, 0, q, jb.DraftTrees(i32([0, 1, 2, 3]), i32(starts), i32(chain(12))), out=guard[1:13])
        assert (guard[0] == 5).all() and (guard[13] == 5).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_strides(dtype):
    """Queries and outputs inside wider rows, layers as slices of one tensor, heads before tokens."""
    trees = [bush(11), chain(30)]
    base, _ = case(dtype, [70, 33], trees, 2, 2, 64, 16)
    both = torch.stack([base.values[0], base.keys[0], base.values[0]], 1).contiguous()
    cache = jb.KVCache(base.pages, [both[:, 1]], [both[:, 2]])
    n = 41
    wide_q = query(n, 4 + 6, 64, dtype)
    out = torch.full((4, n + 1, 64), 7.0, dtype=DT[dtype], device="cuda")
    got = check(cache, 0, wide_q[:, 3:7], range(2), trees, out=out[:, 1:].transpose(0, 1))
    assert (out[:, 0] == 7).all() and got.stride(0) == 64


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_repeatable_and_on_other_streams(dtype):
    trees = [bush(40, i) for i in range(6)]
    cache, q = case(dtype, [900, 5, 2000, 77, 1300, 640], trees, 3, 2, 128, 16, std=0.5)
    t = draft(range(6), trees)
    want = jb.jb_attend_tree(cache, 0, q, t)
    other = torch.cuda.Stream()
    other.wait_stream(torch.cuda.current_stream())
    for _ in range(3):
        a = jb.jb_attend_tree(cache, 0, q, t)
        b = jb.jb_attend_tree(cache, 0, q, t, stream=other)
        with torch.cuda.stream(other):
            c = jb.jb_attend_tree(cache, 0, q, t, workspace=cache.new_tree_workspace())
        torch.cuda.synchronize()
        assert torch.equal(a, want) and torch.equal(b, want) and torch.equal(c, want)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_one_graph_while_rows_grow(dtype):
    """The graph is captured once; lengths, pages and parents are read when it is replayed."""
    cache, q = case(dtype, [300, 64], [chain(8), chain(8)], 2, 2, 64, 16)
    t = draft([0, 1], [chain(8), chain(8)])
    ws, out = cache.new_tree_workspace(), torch.empty_like(q)
    jb.jb_attend_tree(cache, 0, q, t, out=out, workspace=ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        jb.jb_attend_tree(cache, 0, q, t, out=out, workspace=ws)
    for cut, parents in ((0, [chain(8), chain(8)]), (150, [bush(8), wide(8)]), (292, [wide(8), [-1] * 8])):
        cache.pages.lens.copy_(i32([308 - cut, 72 - min(cut, 60)]))
        t.parents.copy_(i32(parents[0] + parents[1]))
        graph.replay()
        want, tol = reference(cache, 0, q, [0, 1], parents)
        assert ((out.double() - want).abs() <= tol).all()


def test_offsets_past_32_bits():
    """Pages more than 2^32 elements into the pool (fp32: 2^34 bytes), of which few are touched."""
    heads, d, page = 8, 128, 1024
    n_pages = (1 << 32) // (heads * d * page) + 2
    pages = jb.PageTable.empty(1, 2, n_pages, page)
    pages.table[0] = i32([n_pages - 1, n_pages - 2])
    pages.lens.fill_(1100)
    for dtype in ("f32", "bf16"):
        k, v = (torch.empty(n_pages, heads, page, d, dtype=DT[dtype], device="cuda") for _ in range(2))
        for x in (k, v):
            x[-2:].normal_()
        tree = bush(9)
        check(jb.KVCache(pages, [k], [v]), 0, query(9, heads, d, dtype), [0], [tree])
        del k, v
        torch.cuda.empty_cache()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_many_small_trees(dtype):
    """More trees than threads of a CTA, a third of them empty."""
    g = torch.Generator().manual_seed(5)
    n = 400
    sizes = [0 if i % 3 == 1 else int(torch.randint(1, 5, (1,), generator=g)) for i in range(n)]
    trees = [bush(s, i) for i, s in enumerate(sizes)]
    tokens = torch.randint(0, 40, (n,), generator=g).tolist()
    cache, q = case(dtype, tokens, trees, 2, 1, 64, 16)
    check(cache, 0, q, range(n), trees)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_scores_far_apart(dtype):
    """A maximum that rises late, tile after tile, and one that is there at once."""
    trees = [chain(5), chain(5)]
    cache, _ = case(dtype, [1000, 1000], trees, 1, 1, 64, 16)
    q = torch.ones(10, 1, 64, dtype=DT[dtype], device="cuda")
    for r in range(2):
        for t in range(1005):
            page, slot = int(cache.pages.table[r, t // 16]), t % 16
            cache.keys[0][page, 0, slot] = (t if r == 0 else 1005 - t) / 64.0
    check(cache, 0, q, range(2), trees, scale=0.5)


LARGE = [bush(200, 3, 2), chain(5), wide(129), bush(256, 1), chain(140), [-1]]   # more than 128 rows a tree on average


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("group,d,page,layout", [(1, 64, 16, "hnd"), (1, 128, 48, "nhd"), (3, 80, 32, "hnd"), (2, 128, 16, "hnd"), (1, 256, 16, "nhd")])
def test_blocks_of_large_trees(dtype, group, d, page, layout):
    """Blocks that are full, half empty and of one row, some of which have no rows for the second half of a block."""
    cache, q = case(dtype, [150, 64, 1, 0, 333, 40], LARGE, 2, group, d, page, layout)
    check(cache, 0, q, range(6), LARGE)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("window,softcap,bias", [(3, 0.0, False), (100, 20.0, False), (0, 3.0, False), (0, 0.0, True), (130, 5.0, True)])
def test_large_trees_with_windows_caps_and_biases(dtype, window, softcap, bias):
    cache, _ = case(dtype, [150, 64, 1, 0, 333, 40], LARGE, 2, 2, 64, 16)
    q = query(sum(map(len, LARGE)), 4, 64, dtype, std=4.0)
    slopes = 2.0 ** -torch.arange(1, 5, device="cuda").float() if bias else None
    check(cache, 0, q, range(6), LARGE, window=window, softcap=softcap, slopes=slopes)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_large_trees_with_gaps(dtype):
    """Missing pages, invalid chains and rows, and values that are not finite in nodes that few see."""
    trees = [list(t) for t in LARGE]
    trees[0][150], trees[4][77] = 151, -2
    cache, q = case(dtype, [150, 64, 1, 0, 333, 40], trees, 2, 1, 128, 16)
    cache.pages.table[0, 4] = -1
    cache.pages.table[3, 9] = -1
    cache.pages.table[4, 3:5] = -1
    rows = [0, 1, 2, 3, 4, 9]
    clean = check(cache, 0, q, rows, trees, out=torch.full_like(q, math.nan))
    base, first = 64, len(trees[0])                     # the chain of five: its last node alone sees itself
    cache.values[0][int(cache.pages.table[1, (base + 4) // 16]), :, (base + 4) % 16] = math.inf
    got = jb.jb_attend_tree(cache, 0, q, draft(rows, trees))
    same = [j for j in range(len(q)) if j != first + 4]
    assert torch.equal(got[same], clean[same]) and not torch.isfinite(got[first + 4]).any()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("group", [1, 3, 8])
def test_large_trees_queries_in_wider_rows(dtype, group):
    """Queries of part of a row's heads, outputs likewise, several streams, one cache."""
    trees = [bush(180), chain(130), bush(250, 2)]
    cache, _ = case(dtype, [70, 200, 9], trees, 2, group, 128, 16)
    n = sum(map(len, trees))
    wide_q = query(n, 2 * group + 3, 128, dtype)
    q = wide_q[:, 2:2 + 2 * group]
    want = check(cache, 0, q.contiguous(), range(3), trees)
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    got = []
    for _ in range(4):
        for s in streams:
            with torch.cuda.stream(s):
                out = torch.full((n, 2 * group + 1, 128), 7.0, dtype=q.dtype, device="cuda")
                jb.jb_attend_tree(cache, 0, q, draft(range(3), trees), out=out[:, 1:])
                got.append(out)
    torch.cuda.synchronize()
    assert all(torch.equal(o[:, 1:], want) and (o[:, 0] == 7).all() for o in got)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("tree", [bush(20), bush(200)], ids=["small", "large"])
def test_broadcast_and_transposed_queries(dtype, tree):
    """One query for all nodes, one for all heads, and heads before nodes."""
    n = len(tree)
    cache, q = case(dtype, [90], [tree], 2, 2, 128, 16)
    for view in (q[:1].expand(n, 4, 128), q[:, :1].expand(n, 4, 128), query(n * 4, 1, 128, dtype).view(4, n, 128).transpose(0, 1)):
        want = check(cache, 0, view.contiguous(), [0], [tree])
        assert torch.equal(jb.jb_attend_tree(cache, 0, view, draft([0], [tree])), want)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("length", [(1 << 31) - 16, (1 << 31) - 20, (1 << 31) - 49])
def test_rows_that_end_at_2_to_the_31(dtype, length):
    """A window over the last tokens of the longest row: the tile of the last ones ends where positions leave 31 bits. Pages
    further back are missing, places without a token and siblings' values hold NaN."""
    tree, window, page = [-1, 0, 0, 1, 1, 0, 5], 300, 16
    tokens = 400                                                          # that there are pages for
    row_pages, first = (1 << 27) - 1, -(-length // page) - tokens // page
    shift = first * page                                                  # the same tokens as a short row
    small, q = case(dtype, [length - shift - len(tree)], [tree], 2, 1, 64, page)
    pages = jb.PageTable.empty(1, row_pages, small.pages.refs.shape[0], page)
    n = int((small.pages.table[0] >= 0).sum())
    pages.table[0, first:first + n] = small.pages.table[0, :n]
    pages.refs.copy_(small.pages.refs)
    pages.lens.fill_(length)
    cache = jb.KVCache(pages, small.keys, small.values)
    want, tol = reference(small, 0, q, [0], [tree], window=window)
    got = jb.jb_attend_tree(cache, 0, q, draft([0], [tree]), window=window)
    assert torch.isfinite(got).all() and ((got.double() - want).abs() <= tol).all()
    leaf = length - shift - 1                                             # the last node: itself alone sees it
    small.values[0][int(small.pages.table[0, leaf // page]), :, leaf % page] = math.nan
    hurt = jb.jb_attend_tree(cache, 0, q, draft([0], [tree]), window=window)
    assert torch.equal(hurt[:-1], got[:-1]) and torch.isnan(hurt[-1]).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_large_products_under_a_small_scale(dtype):
    """Products of -3.1e38 by a scale of 2^-120 are scores of -232, as good as any others."""
    trees = [chain(3), chain(1)]
    cache, _ = case(dtype, [70, 0], trees, 1, 1, 64, 16, spare=0)
    q = torch.full((4, 1, 64), 2.0**61, dtype=DT[dtype], device="cuda")
    cache.keys[0].copy_(torch.where(torch.isnan(cache.keys[0]), cache.keys[0], torch.full_like(cache.keys[0], -1.8125 * 2.0**60)))
    check(cache, 0, q, range(2), trees, scale=2.0**-120)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("scale", [1.0, 4.0])
def test_scores_beyond_2e38_count_as_infinite(dtype, scale):
    """Products of -3.0e38 leave fp32 with the factor that makes powers of two of exponentials: those positions are not seen, and a
    node that sees no others gets zeros, as single queries have it."""
    trees = [chain(3), chain(2)]
    cache, _ = case(dtype, [130, 20], trees, 1, 1, 64, 16, spare=0)
    q = torch.full((5, 1, 64), 2.0**61, dtype=DT[dtype], device="cuda")
    key = torch.where(torch.isnan(cache.keys[0]), cache.keys[0], torch.full_like(cache.keys[0], -1.75 * 2.0**60))
    for t in range(0, 133, 3):
        key[int(cache.pages.table[0, t // 16]), :, t % 16] = 0.0
    cache.keys[0].copy_(key)
    got = jb.jb_attend_tree(cache, 0, q, draft(range(2), trees), scale=scale)
    one = jb.jb_attend(cache, 0, q, i32([0, 0, 0, 1, 1]), i32([130, 131, 132, 20, 21]), scale=scale)
    assert (got[3:] == 0).all() and (one[3:] == 0).all()
    for j in range(3):
        place = torch.arange(0, 131 + j, 3)
        ids = cache.pages.table[0].cpu()[place // 16].long()
        want = cache.values[0][ids.cuda(), 0, (place % 16).cuda()].double().mean(0)
        tol = 2.0**-20 + (2.0**-16 + 2.0**-8 * want.abs() if dtype == "bf16" else 0)
        assert ((got[j, 0].double() - want).abs() <= tol).all() and ((one[j, 0].double() - want).abs() <= tol).all()


@pytest.mark.parametrize("bad", [math.nan, math.inf])
def test_many_blocks_some_with_values_that_are_not_finite(bad):
    """A CTA works on block after block: what it has to mend in one says nothing of the others."""
    n, heads = 400, 8
    trees = [bush(3 + i % 5, i) for i in range(n)]
    cache, q = case("bf16", [(7 * i) % 50 for i in range(n)], trees, heads, 1, 64, 16)
    clean = check(cache, 0, q, range(n), trees)
    table, lens, first, own = cache.pages.table.cpu(), cache.pages.lens.tolist(), 0, []
    for i, tree in enumerate(trees):
        if i % 7 == 0:                                                    # the tree's last node, which nobody follows
            t = lens[i] - 1
            cache.values[0][int(table[i, t // 16]), :, t % 16] = bad
            own.append(first + len(tree) - 1)
        first += len(tree)
    got = jb.jb_attend_tree(cache, 0, q, draft(range(n), trees))
    others = sorted(set(range(first)) - set(own))
    assert torch.equal(got[others], clean[others]) and not torch.isfinite(got[own]).any()
