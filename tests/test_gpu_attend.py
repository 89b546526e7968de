"""jb_attend against the definition in 64 bits, where it can go wrong: lengths around groups and pages,
empty and invalid queries, heads that share keys, head sizes between the kernels', both layouts, what
unseen places hold, strides, streams, offsets past 32 bits.

Tolerances. With A = sum_t p_t |v_t| (p the exact weights) and S = max_t scale sum_e |q_e k_e|:
* a score is a sum of d products in fp32 and a few roundings: off by at most (d + 16) 2^-23 S (and as
  much again for the cap and the bias, whose operands are below S' = S + bias), which moves every
  weight by that factor, twice (numerator and sum);
* the exponential is good to 2^-21, weights enter bf16 products with 2^-16, the sums of T terms lose at
  most T 2^-23;
* a bf16 result is rounded once, 2^-9 of it (2^-8 allows for the tie).
"""
import math

import pytest
import torch

import paper_2306_10015_gb300 as jb

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def make(dtype, lens, heads, d, page, layout="hnd", spare=2, seed=0, fill=math.nan, layers=1, std=1.0):
    """A cache whose rows hold lens tokens in shuffled pages; every place no token has holds `fill`."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    lens = torch.tensor(lens)
    need = -(-lens // page)
    n_pages, row_pages = int(need.sum()) + spare, max(1, int(need.max())) + 1
    ids = torch.randperm(n_pages, generator=torch.Generator().manual_seed(seed)).int()
    table = torch.full((len(lens), row_pages), -1, dtype=torch.int32)
    at = 0
    for i, k in enumerate(need.tolist()):
        table[i, :k] = ids[at:at + k]
        at += k
    refs = torch.zeros(n_pages, dtype=torch.int32)
    refs[ids[:at].long()] = 1
    shape = (n_pages, heads, page, d) if layout == "hnd" else (n_pages, page, heads, d)
    pools = []
    for _ in range(2 * layers):
        x = torch.randn(shape, generator=g, device="cuda") * std
        x = x.to(DT[dtype])
        x = x if layout == "hnd" else x.transpose(1, 2)
        held = torch.zeros(n_pages, page, dtype=torch.bool)
        for i, n in enumerate(lens.tolist()):
            for j in range(0, n, page):
                held[table[i, j // page], :min(page, n - j)] = True
        x.masked_fill_(~held.cuda()[:, None, :, None], fill)
        pools.append(x)
    pages = jb.PageTable(table.cuda(), lens.int().cuda(), refs.cuda(), page)
    return jb.KVCache(pages, pools[:layers], pools[layers:])


def reference(cache, layer, q, rows, pos, scale=None, softcap=0.0, window=0, slopes=None):
    """(result, tolerance) of every element in 64 bits."""
    n, qh, d = q.shape
    g = qh // cache.heads
    scale = d ** -0.5 if scale is None else scale
    page = cache.pages.page_tokens
    out = torch.zeros(n, qh, d, dtype=torch.float64, device="cuda")
    tol = torch.zeros_like(out)
    table = cache.pages.table.cpu()
    for i, (r, last) in enumerate(zip(rows.tolist(), pos.tolist())):
        if not 0 <= r < table.shape[0] or not 0 <= last < table.shape[1] * page:
            continue
        t = torch.arange(max(0, last - window + 1) if window else 0, last + 1)
        ids = table[r, t // page].long()
        t, ids = t[ids >= 0], ids[ids >= 0]
        if len(t) == 0:
            continue
        k = cache.keys[layer][ids.cuda(), :, (t % page).cuda()].double().repeat_interleave(g, 1)     # [T, qh, d]
        v = cache.values[layer][ids.cuda(), :, (t % page).cuda()].double().repeat_interleave(g, 1)
        prod = q[i].double()[None] * k * scale
        x, size = prod.sum(-1), prod.abs().sum(-1).amax(0)
        if softcap:
            x = softcap * torch.tanh(x / softcap)
            size = size + softcap
        if slopes is not None:
            x = x + slopes.double()[None] * (t.cuda() - last).double()[:, None]
            size = size + slopes.double() * float(last - t[0])
        p = torch.softmax(x, 0)
        out[i] = torch.einsum("th,thd->hd", p, v)
        a = torch.einsum("th,thd->hd", p, v.abs())
        rel = 2 * (2 * (d + 16) * 2.0**-23 * size + 2.0**-21) + len(t) * 2.0**-23
        if q.dtype == torch.bfloat16:
            rel = rel + 2.0**-16
        tol[i] = a * rel[:, None] + (2.0**-8 * out[i].abs() if q.dtype == torch.bfloat16 else 0) + 1e-38
    return out, tol


def check(cache, layer, q, rows, pos, **kw):
    got = jb.jb_attend(cache, layer, q, rows, pos, **kw)
    want, tol = reference(cache, layer, q, rows, pos, **{k: v for k, v in kw.items() if k not in ("out", "stream")})
    torch.cuda.synchronize()
    err = (got.double() - want).abs()
    assert torch.isfinite(got).all()
    worst = (err / tol.clamp(min=1e-300)).amax() if err.numel() else 0.0
    assert (err <= tol).all(), f"worst error over tolerance {worst:.3g}"
    return got


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def query(n, heads, d, dtype, seed=1, std=2.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(n, heads, d, generator=g, device="cuda") * std).to(DT[dtype])


LENS = [1, 0, 15, 16, 17, 31, 33, 47, 48, 49, 63, 64, 65, 127, 128, 129, 255, 257, 700]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("page,layout", [(16, "hnd"), (48, "nhd"), (128, "hnd"), (64, "nhd")])
def test_lengths_around_groups_and_pages(dtype, page, layout):
    cache = make(dtype, LENS, 3, 64, page, layout)
    check(cache, 0, query(len(LENS), 3, 64, dtype), i32(range(len(LENS))), cache.pages.lens - 1)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("d", [8, 16, 40, 64, 72, 80, 96, 120, 128, 136, 192, 256])
@pytest.mark.parametrize("group", [1, 3])
def test_head_sizes(dtype, d, group):
    lens = [5, 130, 64]
    cache = make(dtype, lens, 2, d, 32)
    check(cache, 0, query(3, 2 * group, d, dtype), i32(range(3)), cache.pages.lens - 1)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("heads,group", [(1, 1), (4, 2), (2, 4), (1, 5), (2, 7), (1, 8), (3, 9), (1, 16), (1, 27), (1, 64)])
@pytest.mark.parametrize("layout", ["hnd", "nhd"])
def test_shared_heads(dtype, heads, group, layout):
    lens = [3, 200, 77]
    cache = make(dtype, lens, heads, 128, 16, layout)
    check(cache, 0, query(3, heads * group, 128, dtype), i32(range(3)), cache.pages.lens - 1)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("window", [0, 1, 2, 15, 16, 17, 64, 100, 5000])
@pytest.mark.parametrize("softcap,bias", [(0.0, False), (20.0, False), (0.0, True), (5.0, True)])
def test_windows_caps_and_biases(dtype, window, softcap, bias):
    lens = [1, 16, 65, 0, 333]
    cache = make(dtype, lens, 2, 64, 16)
    slopes = 2.0 ** -torch.arange(1, 7, device="cuda").float() if bias else None
    check(cache, 0, query(5, 6, 64, dtype, std=4.0), i32(range(5)), cache.pages.lens - 1, window=window, softcap=softcap, slopes=slopes)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("cap", [1e-3, 0.25, 7.0, 50.0, 3e3, 1e7, 1e25])
def test_caps_keep_small_scores(dtype, cap):
    """Whatever the cap, tanh is good to a few parts in 2^20 of itself: the score moves by no more than that of
    its own size (here 2^-19 of the largest score after the cap), not of the cap's."""
    cache = make(dtype, [200], 2, 64, 16)
    q, rows, pos = query(1, 2, 64, dtype, std=3.0), i32([0]), i32([199])
    got = jb.jb_attend(cache, 0, q, rows, pos, softcap=cap)
    ids = cache.pages.table[0, torch.arange(200, device="cuda") // 16].long()
    k, v = (x[0][ids, :, torch.arange(200, device="cuda") % 16].double() for x in (cache.keys, cache.values))
    prod = q[0].double()[None] * k / 8.0
    x = cap * torch.tanh(prod.sum(-1) / cap)
    p = torch.softmax(x, 0)
    want, size = torch.einsum("th,thd->hd", p, v), torch.einsum("th,thd->hd", p, v.abs())
    rel = 2 * (80 * 2.0**-23 * prod.abs().sum(-1).amax(0) + 2.0**-19 * x.abs().amax(0) + 2.0**-21) + 200 * 2.0**-23
    tol = size * (rel[:, None] + (2.0**-16 if dtype == "bf16" else 0)) + (2.0**-8 * want.abs() if dtype == "bf16" else 0)
    assert ((got[0].double() - want).abs() <= tol).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_prompt_tokens_are_queries_of_one_row(dtype):
    cache = make(dtype, [150, 40], 2, 64, 16)
    rows, pos = i32([0] * 150 + [1] * 40), i32(list(range(150)) + list(range(40)))
    check(cache, 0, query(190, 4, 64, dtype), rows, pos)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_queries_that_see_nothing(dtype):
    cache = make(dtype, [40, 20, 7], 2, 64, 16)
    cap = cache.pages.struct.row_pages * 16
    rows, pos = i32([0, -1, 3, 1, 2, 0, 1 << 30, 1]), i32([-1, 5, 5, cap, 6, -2147483648, 3, 2147483647])
    q = query(8, 2, 64, dtype)
    out = torch.full_like(q, math.nan)
    got = check(cache, 0, q, rows, pos, out=out)
    assert got is out and (got[[0, 1, 2, 3, 5, 6, 7]] == 0).all() and (got[4] != 0).any()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_missing_pages_are_not_seen(dtype):
    """An entry of -1 inside a row, and positions past the row's pages (within its table's row)."""
    cache = make(dtype, [160, 33], 2, 64, 16)
    cache.pages.table[0, 3] = -1
    cache.pages.table[0, 7:9] = -1
    check(cache, 0, query(3, 2, 64, dtype), i32([0, 0, 0]), i32([159, 100, 170]), scale=0.3)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("heads,n", [(1, 1), (2, 3)])
def test_long_rows_are_split_and_joined(dtype, heads, n):
    lens = [50_001, 1, 16_384][:n]
    cache = make(dtype, lens, heads, 128, 64, std=0.5)
    check(cache, 0, query(n, heads * 2, 128, dtype), i32(range(n)), cache.pages.lens - 1)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_many_rows(dtype):
    g = torch.Generator().manual_seed(5)
    lens = torch.randint(0, 90, (700,), generator=g).tolist()
    cache = make(dtype, lens, 2, 64, 16)
    check(cache, 0, query(700, 2, 64, dtype), i32(range(700)), cache.pages.lens - 1)


def test_more_queries_than_one_launch_takes():
    cache = make("bf16", [33], 1, 64, 16)
    n = 16_384 + 77
    q = query(3, 1, 64, "bf16")[torch.arange(n, device="cuda") % 3].contiguous()
    pos = (torch.arange(n, device="cuda") % 33).int()
    got = jb.jb_attend(cache, 0, q, torch.zeros(n, dtype=torch.int32, device="cuda"), pos)
    want, tol = reference(cache, 0, q[:99], i32([0] * 99), pos[:99])
    assert ((got[:99].double() - want).abs() <= tol).all()
    again = torch.arange(n, device="cuda") % 99  # the same queries, cut at other places
    assert ((got - got[:99][again]).double().abs() <= 2 * tol[again]).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_large_scores_and_dominant_tokens(dtype):
    """Maxima that rise along the row, by far more than the exponential's range."""
    cache = make(dtype, [300], 1, 64, 16, std=1.0)
    k = cache.keys[0]
    table = cache.pages.table[0].cpu()
    for t in (20, 150, 299):
        k[int(table[t // 16]), 0, t % 16] *= 20.0 + t
    check(cache, 0, query(1, 2, 64, dtype, std=6.0), i32([0]), i32([299]))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_strided_queries_and_outputs_and_interleaved_pages(dtype):
    lens = [70, 9]
    base = make(dtype, lens, 2, 64, 16)
    both = torch.stack([base.keys[0], base.values[0]], 1)  # [pages, 2, heads, tokens, d]
    cache = jb.KVCache(base.pages, [both[:, 0]], [both[:, 1]])
    qkv = query(2, 8, 64, dtype)
    q = qkv[:, 2:6]
    out = torch.zeros(2, 9, 64, dtype=q.dtype, device="cuda")
    check(cache, 0, q, i32([0, 1]), base.pages.lens - 1, out=out[:, 1:5])
    assert (out[:, 0] == 0).all() and (out[:, 5:] == 0).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_results_repeat_and_streams_are_kept(dtype):
    lens = [4000, 3, 900, 0, 2500]
    cache = make(dtype, lens, 4, 128, 16)
    q, rows, pos = query(5, 8, 128, dtype), i32(range(5)), cache.pages.lens - 1
    first = jb.jb_attend(cache, 0, q, rows, pos)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        a = jb.jb_attend(cache, 0, q, rows, pos)
    b = jb.jb_attend(cache, 0, q, rows, pos, stream=s)
    c = jb.jb_attend(cache, 0, q, rows, pos, stream=s.cuda_stream)
    s.synchronize()
    for x in (a, b, c):
        assert torch.equal(first, x)


def test_in_a_graph_lengths_may_change():
    cache = make("bf16", [500, 40], 2, 64, 16)
    q, rows, pos = query(2, 4, 64, "bf16"), i32([0, 1]), i32([10, 10])
    out = torch.empty_like(q)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        jb.jb_attend(cache, 0, q, rows, pos, out=out)
    torch.cuda.current_stream().wait_stream(s)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        jb.jb_attend(cache, 0, q, rows, pos, out=out)
    for p in ([499, 39], [0, -1], [250, 17]):
        pos.copy_(i32(p))
        graph.replay()
        want, tol = reference(cache, 0, q, rows, pos)
        torch.cuda.synchronize()
        assert ((out.double() - want).abs() <= tol).all()


def test_offsets_past_32_bits():
    """Pages whose elements lie beyond 2^32 elements of their tensor."""
    heads, d, page = 32, 128, 16
    n_pages = (1 << 32) // (heads * d * page) + 40
    k = torch.empty(n_pages, heads, page, d, dtype=torch.bfloat16, device="cuda")
    v = torch.empty_like(k)
    k[-30:].normal_()
    v[-30:].normal_()
    table = torch.full((2, 9), -1, dtype=torch.int32)
    table[0, :8] = torch.arange(n_pages - 8, n_pages)
    table[1, :3] = torch.tensor([n_pages - 20, n_pages - 11, n_pages - 30])
    pages = jb.PageTable(table.cuda(), i32([128, 41]), torch.zeros(n_pages, dtype=torch.int32, device="cuda"), page)
    cache = jb.KVCache(pages, [k], [v])
    check(cache, 0, query(2, 32, 128, "bf16"), i32([0, 1]), i32([127, 40]))
    new = query(2, 64, 128, "bf16", seed=9)
    jb.jb_cache_write(cache, 0, new[:, :32], new[:, 32:], i32([0, 1]), i32([100, 47]))
    assert torch.equal(k[n_pages - 8 + 6, :, 4], new[0, :32]) and torch.equal(v[n_pages - 30, :, 15], new[1, 32:])


def test_workspace_on_the_host_is_refused():
    pages = jb.PageTable.empty(1, 2, 2, 16)
    kv = torch.zeros(2, 1, 16, 64, dtype=torch.bfloat16, device="cuda")
    cache = jb.KVCache(pages, [kv], [kv.clone()])
    at = torch.zeros(1, dtype=torch.int32, device="cuda")
    q = torch.zeros(1, 1, 64, dtype=torch.bfloat16, device="cuda")
    size = cache.new_workspace(1).numel()
    for ws in (torch.zeros(size, dtype=torch.uint8), torch.zeros(2 * size, dtype=torch.uint8, device="cuda")[::2]):
        with pytest.raises(ValueError):
            jb.jb_attend(cache, 0, q, at, at, workspace=ws)


def test_groups_of_a_run_of_queries_pass_32_bits():
    """17 queries in a row at the end of a row of 2^31 - 1024 tokens: a thread's run of them has more than 2^31 groups
    of 16. All pages but the last are missing, so no key is copied for the others. The wanted values are those of a
    row that has this page alone."""
    page, row_pages, n = 1024, (1 << 21) - 1, 17 * 128
    kv = torch.randn(2, 1, 1, page, 64, device="cuda").to(torch.bfloat16)
    table = torch.full((1, row_pages), -1, dtype=torch.int32, device="cuda")
    table[0, -1] = 0
    cache = jb.KVCache(jb.PageTable(table, i32([row_pages * page]), i32([1]), page), [kv[0]], [kv[1]])
    short = jb.KVCache(jb.PageTable(i32([[0]]), i32([page]), i32([1]), page), [kv[0]], [kv[1]])
    q, rows = query(n, 1, 64, "bf16"), torch.zeros(n, dtype=torch.int32, device="cuda")
    at = torch.full((n,), -1, dtype=torch.int32)
    at[17 * 40:17 * 41] = page - 1 - 3 * torch.arange(17, dtype=torch.int32)
    first = (row_pages - 1) * page
    got = jb.jb_attend(cache, 0, q, rows, torch.where(at >= 0, at + first, -1).int().cuda())
    want, tol = reference(short, 0, q, rows, at.cuda())
    assert ((got.double() - want).abs() <= tol).all() and (got[17 * 40:17 * 41] != 0).any() and (got[:17 * 40] == 0).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_two_streams_at_the_same_time(dtype):
    """Calls whose rows are split, on one cache from two streams without waiting in between: each stream has its own
    parts to join."""
    cache = make(dtype, [9000, 5, 3000], 2, 128, 16)
    rows, pos = i32([0, 1, 2]), cache.pages.lens - 1
    queries = [query(3, 4, 128, dtype, seed=s) for s in range(20, 26)]
    want = [check(cache, 0, q, rows, pos) for q in queries]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    got = [jb.jb_attend(cache, 0, queries[i % 6], rows, pos, stream=streams[i % 2]) for i in range(120)]
    torch.cuda.synchronize()
    for i, x in enumerate(got):
        assert torch.equal(x, want[i % 6])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_kept_workspaces_grow(dtype):
    """Few query heads, then more of them (a larger workspace on the same stream), and few again."""
    cache = make(dtype, [6000, 700], 2, 128, 16)
    rows, pos = i32([0, 1]), cache.pages.lens - 1
    first = {}
    for group in (1, 16, 1, 2, 16, 9, 1):
        got = check(cache, 0, query(2, 2 * group, 128, dtype), rows, pos)
        assert torch.equal(first.setdefault(group, got), got)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("length", [40, 5000])
@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan])
def test_values_that_are_not_finite_and_seen(dtype, length, bad):
    """They reach their own element of the heads that read them, and nothing else; in fp32 an infinity stays one. The
    token's weight is made large, so that it is not lost in the sum."""
    cache = make(dtype, [length], 2, 64, 16)
    q, rows, pos = query(1, 6, 64, dtype), i32([0]), i32([length - 1])
    t = length // 2
    page = int(cache.pages.table[0, t // 16])
    cache.keys[0][page, 1, t % 16] = q[0, 3:].mean(0)
    want, tol = reference(cache, 0, q, rows, pos)
    cache.values[0][page, 1, t % 16, 17] = bad
    got = jb.jb_attend(cache, 0, q, rows, pos)
    hit = torch.zeros(1, 6, 64, dtype=torch.bool, device="cuda")
    hit[0, 3:, 17] = True
    assert not torch.isfinite(got[hit]).any()
    if dtype == "f32" and not math.isnan(bad):
        assert (got[hit] == bad).all()
    assert ((got.double() - want).abs() <= tol)[~torch.isnan(want) & ~hit].all() and torch.isfinite(got[~hit]).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("length", [40, 5000])
def test_keys_that_are_not_finite_and_seen(dtype, length):
    """A score of +inf or NaN gives NaN, one of -inf leaves its token out, and where all are -inf nothing is seen."""
    cache = make(dtype, [length], 2, 64, 16)
    q, rows, pos = query(1, 4, 64, dtype), i32([0]), i32([length - 1])
    q[0, 2:, 5] = q[0, 2:, 5].abs() + 0.5
    t = length // 3
    page = int(cache.pages.table[0, t // 16])
    clean, tol = reference(cache, 0, q, rows, pos)
    for bad in (math.nan, math.inf):
        cache.keys[0][page, 1, t % 16, 5] = bad
        got = jb.jb_attend(cache, 0, q, rows, pos)
        assert torch.isnan(got[0, 2:]).all() and ((got.double() - clean).abs() <= tol)[0, :2].all()
    cache.keys[0][page, 1, t % 16, 5] = -math.inf
    got = jb.jb_attend(cache, 0, q, rows, pos)[0, 2:].double()
    others = torch.arange(length, device="cuda")
    others = others[others != t]
    ids = cache.pages.table[0, others // 16].long()
    k, v = (x[0][ids, 1, others % 16].double() for x in (cache.keys, cache.values))
    prod = q[0, 2:].double()[:, None] * k / 8.0
    p = torch.softmax(prod.sum(-1), -1)
    size = prod.abs().sum(-1).amax(1, keepdim=True)
    rel = 2 * (2 * 80 * 2.0**-23 * size + 2.0**-21) + length * 2.0**-23 + (2.0**-16 if dtype == "bf16" else 0)
    assert ((got - p @ v).abs() <= (p @ v.abs()) * rel + (2.0**-8 * (p @ v).abs() if dtype == "bf16" else 0)).all()
    cache.keys[0][:, 1, :, 5] = -math.inf
    got = jb.jb_attend(cache, 0, q, rows, pos)
    assert (got[0, 2:] == 0).all() and ((got.double() - clean).abs() <= tol)[0, :2].all()
