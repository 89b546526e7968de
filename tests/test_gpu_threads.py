"""Host threads that share a stream, a table of 4-bit weights and a cache, whose workspaces are the ones kept for the stream."""
import threading

import pytest
import torch

import paper_2306_10015_gb300 as jb
from test_gpu_attend import DT, i32, query
from test_gpu_q4_matmul import weights
from test_gpu_tree import bush, case, chain, draft

pytestmark = pytest.mark.gpu


def side_by_side(*work):
    """Each of the functions in a thread of its own, all starting together; what they raise."""
    start, failed = threading.Barrier(len(work)), []

    def run(f):
        try:
            start.wait()
            f()
        except Exception as e:  # noqa: BLE001
            failed.append(e)
    threads = [threading.Thread(target=run, args=(f,)) for f in work]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert not failed, failed[0]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_products(dtype):
    table, got = weights(2100, 2048), [[], [], []]
    x = [torch.randn(n, 2048, device="cuda").to(DT[dtype]) for n in (33, 64, 24)]
    want = [jb.jb_q4_matmul(table, 0, v, 2100) for v in x]
    torch.cuda.synchronize()

    def work(i):
        for _ in range(150):
            got[i].append(jb.jb_q4_matmul(table, 0, x[i], 2100))
    side_by_side(*(lambda i=i: work(i) for i in range(3)))
    assert all(torch.equal(y, want[i]) for i in range(3) for y in got[i])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_trees_of_one_cache(dtype):
    trees = [[bush(40, 1), chain(9)], [bush(150, 2), bush(33, 3)]]
    cache, _ = case(dtype, [900, 77, 1300, 640], trees[0] + trees[1], 3, 2, 64, 16)
    t = [draft([0, 1], trees[0]), draft([2, 3], trees[1])]
    q = [query(49, 6, 64, dtype), query(183, 6, 64, dtype, seed=1)]
    want, got = [jb.jb_attend_tree(cache, 0, q[i], t[i]) for i in range(2)], [[], []]
    torch.cuda.synchronize()

    def work(i):
        for _ in range(100):
            got[i].append(jb.jb_attend_tree(cache, 0, q[i], t[i]))
    side_by_side(lambda: work(0), lambda: work(1))
    assert all(torch.equal(y, want[i]) for i in range(2) for y in got[i])


def test_rows_of_one_cache():
    """Each thread appends to its rows and keeps paths of them, over and over; pages that one gives back the other gets."""
    torch.cuda.synchronize()
    pages = jb.PageTable.empty(4, 80, 320, 16)
    cache = jb.KVCache(pages, [torch.zeros(320, 2, 16, 64, device="cuda") for _ in range(2)], [torch.zeros(320, 2, 16, 64, device="cuda") for _ in range(2)])
    none = jb.Rotation(torch.zeros(32, dtype=torch.int64, device="cuda"))
    tree = bush(100, 4)
    path, j = [], 99
    while j >= 0:
        path.append(j)
        j = tree[j]
    path, status, told = path[::-1], [[], []], [[], []]
    index = torch.arange(100, dtype=torch.int32, device="cuda")

    def work(i):
        rows = i32([2 * i, 2 * i + 1])
        both, leaves, hundreds = draft([2 * i, 2 * i + 1], [tree, tree]), i32([99, 99]), i32([100, 100])
        row_of = rows.repeat_interleave(100)
        for step in range(30):
            k = [torch.randn(200, 2, 64, device="cuda") for _ in range(2)]
            base = pages.lens[rows.long()].clone()
            status[i].append(jb.jb_cache_reserve(cache, rows, hundreds))
            pos = (base[:, None] + index[None]).flatten()
            for layer in range(2):
                jb.jb_cache_append(cache, layer, None, k[layer], k[layer] + 1, row_of, pos, none)
            status[i].append(jb.jb_cache_keep(cache, both, leaves))
            told[i].append([x.view(2, 100, 2, 64)[:, path] for x in k])
    side_by_side(lambda: work(0), lambda: work(1))
    for i in range(2):
        assert all(s.item() == 0 for s in status[i])
        for r in range(2):
            row, n = 2 * i + r, 30 * len(path)
            assert pages.lens[row].item() == n
            at = torch.arange(n, device="cuda")
            ids = pages.table[row].long()[at // 16]
            for layer in range(2):
                want = torch.cat([step[layer][r] for step in told[i]])
                assert torch.equal(cache.keys[layer][ids, :, at % 16], want) and torch.equal(cache.values[layer][ids, :, at % 16], want + 1)
