"""jb_cache_keep against a plain model of the pages (that of test_gpu_cache.py). All values are compared exactly."""
import random

import pytest
import torch

import paper_2306_10015_gb300 as jb
from test_gpu_cache import Both, i32
from test_gpu_tree import bush, chain, draft, path_to, wide

pytestmark = pytest.mark.gpu


def keep_model(m, rows, trees, leaves):
    """Status and the moves: ((page, place) from, to)."""
    moves, ends = [], []
    if len(set(rows)) < len(rows):
        return -1, []
    for r, tree, leaf in zip(rows, trees, leaves):
        if not 0 <= r < len(m.rows) or len(tree) > 256 or m.lens[r] < len(tree) or not -1 <= leaf < len(tree):
            return -1, []
        path = path_to(tree, leaf)
        if path is None:
            return -1, []
        base = m.lens[r] - len(tree)
        for k, j in enumerate(path):
            if j == k:
                continue
            a, b = m.rows[r][(base + j) // m.page], m.rows[r][(base + k) // m.page]
            if m.refs[b] != 1:
                return -1, []
            moves.append((a, (base + j) % m.page, b, (base + k) % m.page))
        ends.append((r, base + len(path)))
    for r, end in ends:
        need = -(-end // m.page)
        for p in m.rows[r][need:]:
            m.refs[p] -= 1
        m.rows[r], m.lens[r] = m.rows[r][:need], end
    return 0, moves


def keep(both, rows, trees, leaves, **kw):
    want, moves = keep_model(both.model, rows, trees, leaves)
    old = [x.clone() for x in both.want]
    for a, i, b, j in moves:
        for x, y in zip(both.want, old):
            x[b, :, j] = y[a, :, i]
    assert jb.jb_cache_keep(both.cache, draft(rows, trees), i32(leaves), **kw).item() == want
    both.same()
    return want


@pytest.mark.parametrize("layout", ["hnd", "nhd"])
@pytest.mark.parametrize("dtype,heads,d,page", [(torch.float32, 3, 8, 16), (torch.bfloat16, 5, 64, 48), (torch.bfloat16, 1, 136, 16), (torch.float32, 2, 4, 32)])
def test_paths(layout, dtype, heads, d, page):
    both = Both(n_rows=5, row_pages=12, n_pages=60, page=page, heads=heads, d=d, layers=3, dtype=dtype, layout=layout)
    both.reserve([0, 1, 2, 3], [70, 33, 16, 1])
    assert keep(both, [2, 0, 3, 1], [chain(16), bush(40), [-1], wide(30)], [9, 39, 0, 29]) == 0
    assert keep(both, [0, 1], [wide(20), bush(5)], [-1, 4]) == 0
    assert keep(both, [1], [chain(both.model.lens[1])], [-1]) == 0           # nothing is left of the row
    assert both.model.lens[1] == 0
    both.reserve([1], [25])
    assert keep(both, [1], [[-1] * 25], [24]) == 0
    assert keep(both, [], [], []) == 0


def test_a_whole_row_of_256():
    both = Both(n_rows=2, row_pages=24, n_pages=48, page=16)
    both.reserve([0, 1], [256, 300])
    odd = [-1] + [max(0, 2 * ((j - 1) // 2) - 1) if j % 2 else j - 1 for j in range(1, 256)]
    assert keep(both, [1, 0], [bush(256, 3), odd], [255, 255]) == 0
    both.reserve([0], [200])
    assert keep(both, [0], [chain(200)], [199]) == 0                         # nothing moves


def test_all_random():
    r = random.Random(1)
    both = Both(n_rows=6, row_pages=10, n_pages=70, page=16, layers=2)
    for step in range(40):
        rows = r.sample(range(6), r.randint(1, 6))
        both.reserve(rows, [r.randint(0, 30) if both.model.lens[x] < 100 else 0 for x in rows])
        rows = [x for x in r.sample(range(6), r.randint(1, 6)) if both.model.lens[x]]
        trees = [bush(r.randint(0, both.model.lens[x]), step) for x in rows]
        keep(both, rows, trees, [r.randint(-1, len(t) - 1) for t in trees])


def test_refusals_change_nothing():
    both = Both(n_rows=6, row_pages=20, n_pages=100, page=16)
    both.reserve([0, 1, 2], [50, 20, 300])
    good = ([0], [bush(20)], [19])
    for rows, trees, leaves in (([0, 0], [chain(3), chain(3)], [2, 2]), ([0, 6], [bush(9), chain(1)], [8, 0]), ([0, -1], [bush(9), chain(1)], [8, 0]),
                                ([0, 1], [bush(9), chain(21)], [8, 0]), ([0, 2], [bush(9), chain(257)], [8, 0]), ([0, 1], [bush(9), chain(3)], [8, 3]),
                                ([0, 1], [bush(9), chain(3)], [8, -2]), ([1, 0], [[-1, 2, 1], bush(9)], [2, 8]), ([1, 0], [[-2, 0, 1], bush(9)], [2, 8]),
                                ([1, 0], [[-1, 1, 1], bush(9)], [1, 8])):
        assert keep(both, rows, trees, leaves) == -1
    assert keep(both, [1], [[-1, 2, 0]], [2]) == 0                            # the bad node is not on the path
    # lists that the model has no words for
    for starts in ([3, 1], [-1, 2], [0, 1 << 30], [0, 5], [(1 << 31) - 1, -(1 << 31)]):
        trees = jb.DraftTrees(i32([0]), i32(starts), i32([-1, 0, 1, 2]))
        assert jb.jb_cache_keep(both.cache, trees, i32([0])).item() == -1
        both.same()
    assert keep(both, *good) == 0


def test_pages_of_other_rows():
    """Drafted tokens in a page that another row names are not moved to; what the path leaves where it is may be there."""
    both = Both(n_rows=4, row_pages=8, n_pages=40, page=16)
    both.reserve([0], [40])
    status, copies = both.model.fork([0], [1])
    assert jb.jb_cache_fork(both.cache, i32([0]), i32([1])).item() == status == 0
    for a, b, n in copies:
        for x in both.want:
            x[b, :, :n] = x[a, :, :n]
    both.same()
    assert keep(both, [0], [wide(20)], [19]) == -1                           # places 20 to 31 are in the shared second page
    assert keep(both, [0], [chain(20)], [5]) == 0                            # nothing moves: the row ends in it
    assert keep(both, [1], [wide(8)], [7]) == 0                              # the last page is the row's own


def test_missing_pages():
    both = Both(n_rows=2, row_pages=8, n_pages=40, page=16)
    both.reserve([0], [80])
    page = int(both.pages.table[0, 3])
    both.pages.table[0, 3] = -1
    tree = draft([0], [[-1] * 40])
    for leaf, want in ((20, -1), (39, 0)):                                   # from place 60, missing, and from 79
        before = both.pages.table.clone()
        assert jb.jb_cache_keep(both.cache, tree, i32([leaf])).item() == want
        assert torch.equal(both.pages.table, before) == (want == -1)
    assert both.pages.lens.tolist() == [41, 0] and both.pages.refs[page] == 1  # the page that no row names is not given back


def test_many_layers_and_a_graph():
    """More layers than one launch takes; the graph is replayed after the rows have grown again."""
    both = Both(n_rows=3, row_pages=8, n_pages=24, page=16, heads=1, d=8, layers=130)
    trees, leaves = [bush(12), wide(9)], [11, 8]
    both.reserve([0, 2], [30, 17])
    t, l, status = draft([0, 2], trees), i32(leaves), i32([7])
    keep(both, [0, 2], trees, leaves, status=status)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        jb.jb_cache_keep(both.cache, t, l, status=status)
    for _ in range(3):
        both.reserve([0, 2], [14, 11])
        want, moves = keep_model(both.model, [0, 2], trees, leaves)
        old = [x.clone() for x in both.want]
        for a, i, b, j in moves:
            for x, y in zip(both.want, old):
                x[b, :, j] = y[a, :, i]
        status.fill_(5)
        graph.replay()
        assert status.item() == want == 0
        both.same()


def test_a_row_that_ends_at_2_to_the_31():
    """Its last pages are there, of 48 tokens, so that the row's end is less than a page from where positions leave 31 bits."""
    page, n_pages, heads, d = 48, 16, 2, 8
    row_pages = ((1 << 31) - 1) // page
    pages = jb.PageTable.empty(1, row_pages, n_pages, page)
    length, nodes = row_pages * page - 3, 200
    pages.table[0, row_pages - 8:] = torch.arange(8, dtype=torch.int32, device="cuda")
    pages.refs[:8] = 1
    pages.lens.fill_(length)
    k, v = (torch.randn(n_pages, heads, page, d, device="cuda") for _ in range(2))
    cache = jb.KVCache(pages, [k], [v])
    assert jb.jb_cache_keep(cache, draft([0], [chain(nodes)]), i32([9])).item() == 0
    kept = length - nodes + 10
    left = -(-kept // page) - (row_pages - 8)                             # of the eight pages
    assert pages.lens.tolist() == [kept] and 0 < left < 8
    assert pages.table[0, row_pages - 8:].tolist() == list(range(left)) + [-1] * (8 - left)
    assert pages.refs[:8].tolist() == [1] * left + [0] * (8 - left)
