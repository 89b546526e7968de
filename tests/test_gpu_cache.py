"""The pages of a cache against a plain model of them: rows as lists of page ids, counts, and what
every place of every page holds. All values are compared exactly."""
import random
import threading

import pytest
import torch

import paper_2306_10015_gb300 as jb

pytestmark = pytest.mark.gpu


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


class Model:
    """The definition, on the host."""

    def __init__(self, n_rows, row_pages, n_pages, page):
        self.rows, self.lens = [[] for _ in range(n_rows)], [0] * n_rows
        self.refs, self.page, self.row_pages = [0] * n_pages, page, row_pages

    def free_ids(self):
        return [p for p, r in enumerate(self.refs) if r == 0]

    def reserve(self, rows, tokens):
        if len(set(rows)) < len(rows) or any(not 0 <= r < len(self.rows) or t < 0 for r, t in zip(rows, tokens)):
            return -1
        if any(self.lens[r] + t > self.row_pages * self.page for r, t in zip(rows, tokens)):
            return -1
        need = [-(-(self.lens[r] + t) // self.page) - len(self.rows[r]) for r, t in zip(rows, tokens)]
        free = self.free_ids()
        if sum(need) > len(free):
            return sum(need) - len(free)
        for r, t, k in zip(rows, tokens, need):
            for _ in range(k):
                self.refs[free[0]] = 1
                self.rows[r].append(free.pop(0))
            self.lens[r] += t
        return 0

    def free(self, rows):
        for r in rows:
            if 0 <= r < len(self.rows):
                for p in self.rows[r]:
                    self.refs[p] -= 1
                self.rows[r], self.lens[r] = [], 0

    def fork(self, parents, children):
        """Status and the copies: (from, to, tokens)."""
        n = len(self.rows)
        if len(set(children)) < len(children) or any(not 0 <= r < n for r in parents + children):
            return -1, []
        old, lens, free, copies = [list(r) for r in self.rows], list(self.lens), self.free_ids(), []
        need = sum(a != b and lens[a] % self.page > 0 for a, b in zip(parents, children))
        if need > len(free):
            return need - len(free), []
        for a, b in zip(parents, children):
            if a == b:
                continue
            row, part = list(old[a]), lens[a] % self.page
            if part:
                copies.append((row[-1], free[0], part))
                row[-1] = free.pop(0)
            for p in row:
                self.refs[p] += 1
            for p in old[b]:
                self.refs[p] -= 1
            self.rows[b], self.lens[b] = row, lens[a]
        return 0, copies

    def compact(self):
        live = [p for p, r in enumerate(self.refs) if r > 0]
        n = len(live)
        moves = list(zip([p for p in live if p >= n], [p for p in range(n) if self.refs[p] == 0]))
        to = dict(moves)
        self.rows = [[to.get(p, p) for p in row] for row in self.rows]
        for a, b in moves:
            self.refs[a], self.refs[b] = 0, self.refs[a]
        return n, moves


class Both:
    """A cache on the GPU and its model."""

    def __init__(self, n_rows=6, row_pages=8, n_pages=24, page=16, heads=3, d=8, layers=2, dtype=torch.float32, layout="hnd"):
        self.model = Model(n_rows, row_pages, n_pages, page)
        self.pages = jb.PageTable.empty(n_rows, row_pages, n_pages, page)
        shape = (n_pages, heads, page, d) if layout == "hnd" else (n_pages, page, heads, d)
        g = torch.Generator(device="cuda").manual_seed(3)
        pools = [torch.randint(-99, 99, shape, device="cuda", generator=g).to(dtype) for _ in range(2 * layers)]
        self.pools = [x if layout == "hnd" else x.transpose(1, 2) for x in pools]
        self.want = [x.clone() for x in self.pools]
        self.cache = jb.KVCache(self.pages, self.pools[:layers], self.pools[layers:])

    def same(self):
        torch.cuda.synchronize()
        m = self.model
        table = [r + [-1] * (m.row_pages - len(r)) for r in m.rows]
        assert self.pages.table.tolist() == table
        assert self.pages.lens.tolist() == m.lens
        assert self.pages.refs.tolist() == m.refs
        count = [0] * len(m.refs)
        for r in m.rows:
            for p in r:
                count[p] += 1
        assert count == m.refs
        for got, want in zip(self.pools, self.want):
            assert torch.equal(got, want)

    def reserve(self, rows, tokens):
        assert jb.jb_cache_reserve(self.cache, i32(rows), i32(tokens)).item() == self.model.reserve(rows, tokens)
        self.same()

    def free(self, rows):
        jb.jb_cache_free(self.cache, i32(rows))
        self.model.free(rows)
        self.same()

    def fork(self, parents, children):
        status, copies = self.model.fork(parents, children)
        assert jb.jb_cache_fork(self.cache, i32(parents), i32(children)).item() == status
        for a, b, n in copies:
            for x in self.want:
                x[b, :, :n] = x[a, :, :n]
        self.same()

    def compact(self):
        n, moves = self.model.compact()
        assert jb.jb_cache_compact(self.cache).item() == n
        for x in self.want:
            if moves:
                a, b = zip(*moves)
                x[list(b)] = x[list(a)]
        self.same()

    def write(self, rows, pos, dtype=None):
        n, x = len(rows), self.pools[0]
        new = torch.randint(-99, 99, (2, n, x.shape[1] + 1, x.shape[3]), device="cuda").to(x.dtype)[:, :, 1:]
        jb.jb_cache_write(self.cache, 1, new[0], new[1], i32(rows), i32(pos))
        m, layers = self.model, len(self.pools) // 2
        for i, (r, p) in enumerate(zip(rows, pos)):
            if 0 <= r < len(m.rows) and 0 <= p < len(m.rows[r]) * m.page:
                self.want[1][m.rows[r][p // m.page], :, p % m.page] = new[0, i]
                self.want[layers + 1][m.rows[r][p // m.page], :, p % m.page] = new[1, i]
        self.same()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("layout", ["hnd", "nhd"])
@pytest.mark.parametrize("page,d", [(16, 8), (48, 40), (128, 256)])
def test_a_life_of_a_cache(dtype, layout, page, d):
    b = Both(page=page, d=d, dtype=dtype, layout=layout)
    b.reserve([2, 0], [page + 3, 1])
    b.reserve([0, 2, 5], [page - 1, 0, 4 * page])
    b.reserve([0], [1])
    b.write([2] * 5 + [0, 5], [0, 1, page - 1, page, page + 2, page, 3 * page])
    b.fork([2, 5, 0], [1, 3, 0])         # a partial page, whole pages only, nothing
    b.write([1, 2], [page + 2, page + 2])
    b.free([5])
    b.compact()
    b.fork([1, 3, 2], [3, 1, 4])         # rows that are both
    b.free([1, 1, 0, 9, -2])             # twice, and out of range
    b.compact()
    b.compact()                          # nothing to move
    b.reserve([0], [2 * page])
    b.free(list(range(6)))
    b.compact()


@pytest.mark.parametrize("seed", range(6))
def test_random_operations(seed):
    g = random.Random(seed)
    n_rows, n_pages = g.choice([(5, 20), (40, 300), (17, 64)])
    b = Both(n_rows=n_rows, row_pages=9, n_pages=n_pages, page=g.choice([16, 32]), heads=g.choice([1, 4]), layout=g.choice(["hnd", "nhd"]),
             dtype=g.choice([torch.float32, torch.bfloat16]))
    for _ in range(40):
        some = g.sample(range(n_rows), g.randint(1, n_rows))
        op = g.choice(["reserve", "reserve", "free", "fork", "fork", "compact", "write"])
        if op == "reserve":
            b.reserve(some, [g.choice([0, 1, 5, 16, 33, g.randint(0, 100)]) for _ in some])
        elif op == "free":
            b.free(some[:2])
        elif op == "fork":
            b.fork([g.randrange(n_rows) for _ in some], some)
        elif op == "compact":
            b.compact()
        else:
            at = sorted({(r, g.randint(-2, 200)) for r in some for _ in range(3)})
            # rows that share a page may name the same place, and such tokens race: one of them is kept
            m = b.model
            place = lambda r, q: (m.rows[r][q // m.page], q % m.page) if 0 <= q < len(m.rows[r]) * m.page else (r, q, "none")  # noqa: E731
            at = list({place(r, q): (r, q) for r, q in at}.values())
            b.write([r for r, _ in at] + [-1, n_rows], [p for _, p in at] + [3, 3])


def test_what_cannot_be_done_changes_nothing():
    b = Both()
    b.reserve([0, 1, 2], [100, 37, 128])
    b.reserve([3, 4], [128, 128])        # too few pages
    b.reserve([3, 3], [1, 1])            # listed twice
    b.reserve([3, 6], [1, 1])            # no such row
    b.reserve([3, -1], [1, 1])
    b.reserve([3, 4], [1, -1])
    b.reserve([2, 3], [1, 1])            # past the table's row
    b.reserve([3], [2147483647])
    b.reserve([3, 4], [16 * 8 - 16, 16])
    b.fork([0, 1], [5, 5])
    b.fork([0, 6], [3, 4])
    b.fork([0, 1], [3, -1])
    b.fork([0, 1, 0], [3, 4, 5])         # too few pages for three copies
    b.reserve([], [])
    b.fork([], [])


@pytest.mark.parametrize("n_pages", [1, 31, 16_384, 16_385, 131_101, 1_000_003])
def test_many_pages(n_pages):
    """One CTA and a cluster of them rank the same pages, in tables whose rows are long."""
    pages = jb.PageTable.empty(4, n_pages, n_pages, 16)
    k = torch.zeros(n_pages, 1, 16, 4, device="cuda") + torch.arange(n_pages, device="cuda").float()[:, None, None, None]
    cache = jb.KVCache(pages, [k], [k.clone()])
    some = torch.randperm(n_pages, device="cuda")[: max(1, n_pages // 3)].sort()[0].int()
    pages.refs[some.long()] = 1
    pages.table[0, : len(some)] = some
    pages.lens[0] = 16 * len(some)
    free = (pages.refs == 0).nonzero().flatten()
    want = len(free) // 2
    assert jb.jb_cache_reserve(cache, i32([1, 2]), i32([16 * (want // 3), 16 * (want - want // 3)])).item() == 0
    got = torch.cat([pages.table[1, : want // 3], pages.table[2, : want - want // 3]])
    assert torch.equal(got.long(), free[:want])
    assert (pages.table[1, want // 3:] == -1).all() and pages.lens.tolist()[1:3] == [16 * (want // 3), 16 * (want - want // 3)]
    jb.jb_cache_free(cache, i32([0]))
    live, rows = int((pages.refs > 0).sum()), pages.table.clone()
    values = k[:, 0, 0, 0].clone()
    assert jb.jb_cache_compact(cache).item() == live
    assert (pages.refs[:live] == 1).all() and (pages.refs[live:] == 0).all()
    now = pages.table.clone()
    held = rows >= 0
    assert torch.equal(held, now >= 0)
    assert torch.equal(k[now[held].long(), 0, 0, 0], values[rows[held].long()])
    assert torch.equal(cache.values[0][now[held].long(), 0, 15, 3], values[rows[held].long()])
    kept = held & (rows < live)
    assert torch.equal(now[kept], rows[kept])


def test_more_pages_asked_for_than_32_bits_count():
    """Rows whose tables are long: the number that is missing is exact, or the largest there is."""
    n, row_pages = 3, 1 << 27                              # 1.6 GB of table, rows of 2^31 - 16 tokens
    pages = jb.PageTable(torch.full((n, row_pages - 1), -1, dtype=torch.int32, device="cuda"), torch.zeros(n, dtype=torch.int32, device="cuda"),
                         torch.zeros(100, dtype=torch.int32, device="cuda"), 16)
    most = 16 * (row_pages - 1)
    assert jb.jb_cache_reserve(pages, i32([0, 1]), i32([most, 17])).item() == row_pages - 1 + 2 - 100
    assert jb.jb_cache_reserve(pages, i32([0, 1, 2]), i32([most, most, most])).item() == 3 * (row_pages - 1) - 100
    assert jb.jb_cache_reserve(pages, i32([0, 1]), i32([most, most + 1])).item() == -1
    assert pages.lens.tolist() == [0, 0, 0] and (pages.refs == 0).all()


def test_many_listed_rows():
    """As many rows as one call takes, forked from one another."""
    n = 16_384
    pages = jb.PageTable.empty(n + 1, 2, 2 * n + 2, 16)
    k = torch.zeros(2 * n + 2, 1, 16, 4, device="cuda")
    cache = jb.KVCache(pages, [k], [k.clone()])
    assert jb.jb_cache_reserve(cache, i32([n]), i32([19])).item() == 0
    k[1, 0, :3] = 7.0
    assert jb.jb_cache_fork(cache, torch.full((n,), n, dtype=torch.int32, device="cuda"), torch.arange(n, dtype=torch.int32, device="cuda")).item() == 0
    assert (pages.table[:, 0] == 0).all() and pages.refs[0].item() == n + 1
    assert torch.equal(pages.table[:n, 1], torch.arange(2, n + 2, device="cuda").int())
    assert (k[2:n + 2, 0, :3] == 7).all() and (k[2:n + 2, 0, 3:] == 0).all() and (k[n + 2:] == 0).all()
    rows = torch.arange(n, dtype=torch.int32, device="cuda")
    assert jb.jb_cache_reserve(cache, rows, torch.full_like(rows, 14)).item() == -1       # 33 tokens in 2 pages
    assert jb.jb_cache_reserve(cache, rows, torch.full_like(rows, 13)).item() == 0
    assert (pages.lens[:n] == 32).all()
    jb.jb_cache_free(cache, torch.arange(n + 1, dtype=torch.int32, device="cuda"))
    assert (pages.table == -1).all() and (pages.refs == 0).all() and (pages.lens == 0).all()


@pytest.mark.parametrize("layers", [1, 127, 129])
def test_many_layers(layers):
    b = Both(layers=layers) if layers > 1 else None
    if b is None:
        b = Both(layers=2)
        b.cache = jb.KVCache(b.pages, b.pools[:1], b.pools[2:3])
        b.want, b.pools = [b.want[0], b.want[2]], [b.pools[0], b.pools[2]]
    b.reserve([0, 1, 2], [37, 20, 5])
    b.fork([0, 1], [3, 4])
    b.free([0, 2])
    b.compact()


def test_other_streams():
    b = Both()
    s = torch.cuda.Stream()
    b.reserve([0, 1], [37, 20])
    torch.cuda.synchronize()
    parents, children, rows = i32([0]), i32([2]), i32([0])
    torch.cuda.synchronize()
    status = jb.jb_cache_fork(b.cache, parents, children, stream=s)
    jb.jb_cache_free(b.cache, rows, stream=s)
    n = jb.jb_cache_compact(b.cache, stream=s.cuda_stream)
    s.synchronize()
    st, copies = b.model.fork([0], [2])
    for a, c, t in copies:
        for x in b.want:
            x[c, :, :t] = x[a, :, :t]
    b.model.free([0])
    live, moves = b.model.compact()
    for a, c in moves:
        for x in b.want:
            x[c] = x[a]
    assert status.item() == st == 0 and n.item() == live
    b.same()


def test_a_generation_step_in_a_graph():
    """Reserve, write and the row's length as the next position, replayed."""
    b = Both(n_rows=2, row_pages=6, n_pages=12, layers=2)
    rows, one = i32([0, 1]), i32([1, 1])
    new = torch.zeros(2, 3, 8, device="cuda")
    status = i32([9])

    def step():
        pos = b.pages.lens.clone()
        jb.jb_cache_reserve(b.cache, rows, one, status=status)
        jb.jb_cache_write(b.cache, 1, new, new, rows, pos)

    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        step()
    torch.cuda.current_stream().wait_stream(s)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in range(1, 40):
        new.fill_(i)
        graph.replay()
    torch.cuda.synchronize()
    assert status.item() == 0 and b.pages.lens.tolist() == [40, 40]
    for r in range(2):
        ids = b.pages.table[r, :3].long()
        assert b.pools[1][ids].transpose(1, 2).reshape(48, 3, 8)[:40, 0, 0].tolist() == [float(i) for i in range(40)]


def test_long_and_longer_lists_at_the_same_time():
    """Host threads whose lists need different amounts of shared memory, above what a launch has by default: each call
    is legal by itself, and so they are side by side."""
    n_rows = 40_000

    def work(n, rounds, errors):
        try:
            stream = torch.cuda.Stream()
            with torch.cuda.stream(stream):
                pages = jb.PageTable.empty(n_rows, 1, 64, 16)
                rows, none, status = torch.arange(n, dtype=torch.int32, device="cuda"), torch.zeros(n, dtype=torch.int32, device="cuda"), i32([7])
                stream.synchronize()
                for _ in range(rounds):
                    jb.jb_cache_reserve(pages, rows, none, status=status)
                stream.synchronize()
                assert status.item() == 0
        except Exception as e:  # noqa: BLE001
            errors.append(e)

    errors = []
    threads = [threading.Thread(target=work, args=(n, 3000, errors)) for n in 2 * (12_300, 13_500, 14_700, 16_384)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not errors, errors[0]


def test_forks_of_unlike_length_and_two_caches_at_the_same_time():
    """A kept workspace that has to grow between calls, and forks, frees and compactions of two caches from two
    streams without waiting in between."""
    caches = [Both(n_rows=64, row_pages=4, n_pages=200, layers=2) for _ in range(2)]
    for b in caches:
        b.reserve([0, 1, 2], [37, 20, 50])
        b.fork([0], [3])
        b.fork([0, 1, 2] * 15, list(range(4, 49)))
        b.free(list(range(4, 30)))
        b.compact()
        b.fork([1, 2], [50, 51])
    lists = [(i32([0, 1, 2]), i32([10, 11, 12])), (i32([2] * 20), i32(list(range(10, 30))))]
    gone = i32(list(range(10, 20)))
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for turn in range(6):
        for b, s in zip(caches, streams):
            jb.jb_cache_fork(b.cache, *lists[turn % 2], stream=s)
            jb.jb_cache_free(b.cache, gone, stream=s)
            jb.jb_cache_compact(b.cache, stream=s)
    torch.cuda.synchronize()
    for b in caches:
        for turn in range(6):
            status, copies = b.model.fork(*[x.tolist() for x in lists[turn % 2]])
            for a, c, n in copies:
                for x in b.want:
                    x[c, :, :n] = x[a, :, :n]
            b.model.free(list(range(10, 20)))
            _, moves = b.model.compact()
            for x in b.want:
                if moves:
                    a, c = zip(*moves)
                    x[list(c)] = x[list(a)]
        b.same()
