"""What the calls on drafted tokens and the products with 4-bit weights refuse, before anything touches CUDA. The device
addresses here are never dereferenced: every call returns an error or is a no-op."""
import ctypes as C

import numpy as np
import pytest

from test_answer_host import BAD_LAYERS, BAD_PAGES, DTYPE, FAKE, INV, MIS, Launches, layer, on_device, p, pages

FAR = FAKE + (1 << 32)   # past the layer's keys and values


@pytest.fixture(scope="module")
def jb():
    from paper_2306_10015_gb300 import build
    build.build()
    import paper_2306_10015_gb300 as pkg
    pkg.lib()
    return pkg


def trees(jb, **kw):
    v = dict(rows=FAKE, starts=FAKE, parents=FAKE, n=2, n_nodes=9)
    v.update(kw)
    return jb.jb_trees(*v.values())


BAD_TREES = [(dict(rows=0), INV), (dict(starts=0), INV), (dict(parents=0), INV), (dict(n=-1), INV), (dict(n=16385), INV), (dict(n_nodes=-1), INV),
             (dict(rows=FAKE + 2), MIS), (dict(starts=FAKE + 1), MIS), (dict(parents=FAKE + 3), MIS)]


def append(jb, q=None, kv=None, rot=None, qp=FAR, qa=256, qb=64, heads=4, out=FAR + (1 << 20), oa=256, ob=64, k=FAR + (2 << 20), ka=128, kb=64,
           v=FAR + (3 << 20), va=128, vb=64, rows=FAKE, pos=FAKE, turns=0, n=1):
    q = C.byref(pages(jb)) if q is None else q
    kv = layer(jb) if kv is None else kv
    rot = jb.jb_rotation(FAKE, 64, 0) if rot is None else rot
    return jb.lib().jb_cache_append(q, C.byref(kv), C.byref(rot), p(qp), qa, qb, heads, p(out), oa, ob, p(k), ka, kb, p(v), va, vb, p(rows), p(pos),
                                    p(turns), n, None)


def attend(jb, q=None, kv=None, scores=None, t=None, qp=FAR, qa=256, qb=64, heads=4, out=FAR + (1 << 20), oa=256, ob=64, ws=FAKE, size=1 << 40):
    q = C.byref(pages(jb)) if q is None else q
    kv = layer(jb) if kv is None else kv
    s = jb.jb_scores(0.125, 0.0, 0, None) if scores is None else scores
    t = trees(jb) if t is None else t
    return jb.lib().jb_attend_tree(q, C.byref(kv), C.byref(s), C.byref(t), p(qp), qa, qb, heads, p(out), oa, ob, p(ws), size, None)


def keep(jb, q=None, kv=None, n_layers=1, t=None, leaves=FAKE, status=FAKE, ws=FAKE, size=1 << 40):
    q = C.byref(pages(jb)) if q is None else q
    kv = layer(jb) if kv is None else kv
    t = trees(jb) if t is None else t
    return jb.lib().jb_cache_keep(q, C.byref(kv), n_layers, C.byref(t), p(leaves), p(status), p(ws), size, None)


def test_bad_page_tables_and_layers(jb):
    for kw, rc in BAD_PAGES:
        q = C.byref(pages(jb, **kw))
        assert append(jb, q) == rc and attend(jb, q) == rc and keep(jb, q) == rc, kw
    for kw, rc in BAD_LAYERS:
        kv = layer(jb, **kw)
        assert append(jb, kv=kv) == rc and attend(jb, kv=kv) == rc and keep(jb, kv=kv) == rc, kw
    two = (jb.jb_kv * 2)(layer(jb), layer(jb, heads=1))
    q, t = C.byref(pages(jb)), trees(jb)
    assert jb.lib().jb_cache_keep(q, two, 2, C.byref(t), p(FAKE), p(FAKE), p(FAKE), 1 << 40, None) == INV
    assert keep(jb, n_layers=0) == INV
    L, s = jb.lib(), jb.jb_scores(0.125, 0.0, 0, None)
    assert L.jb_attend_tree(q, None, C.byref(s), C.byref(t), p(FAR), 256, 64, 4, p(FAKE), 256, 64, p(FAKE), 1 << 40, None) == INV
    assert L.jb_attend_tree(q, C.byref(layer(jb)), None, C.byref(t), p(FAR), 256, 64, 4, p(FAKE), 256, 64, p(FAKE), 1 << 40, None) == INV
    assert L.jb_attend_tree(q, C.byref(layer(jb)), C.byref(s), None, p(FAR), 256, 64, 4, p(FAKE), 256, 64, p(FAKE), 1 << 40, None) == INV


def test_bad_trees(jb):
    for kw, rc in BAD_TREES:
        t = trees(jb, **kw)
        assert attend(jb, t=t) == rc and keep(jb, t=t) == rc, kw
        assert jb.lib().jb_cache_keep_workspace(C.byref(t)) == 0
    assert attend(jb, t=trees(jb, n=0, rows=0, starts=0), qp=0) == 0
    assert attend(jb, t=trees(jb, n_nodes=0, parents=0), qp=0) == 0
    assert jb.lib().jb_cache_keep_workspace(None) == 0
    need = jb.lib().jb_cache_keep_workspace(C.byref(trees(jb)))
    assert need >= 9 * 16 + 2 * 4
    for kw, rc in ((dict(leaves=0), INV), (dict(leaves=FAKE + 2), MIS), (dict(status=0), INV), (dict(status=FAKE + 1), MIS), (dict(ws=0), INV),
                   (dict(ws=FAKE + 8), MIS), (dict(size=need - 1), INV)):
        assert keep(jb, **kw) == rc, kw


def test_bad_tree_attention(jb):
    s = lambda *a: jb.jb_scores(*a)  # noqa: E731
    inf, nan = float("inf"), float("nan")
    need = jb.lib().jb_attend_tree_workspace(C.byref(layer(jb)))
    assert need > 0 and jb.lib().jb_attend_tree_workspace(None) == 0 and jb.lib().jb_attend_tree_workspace(C.byref(layer(jb, head_dim=264))) == 0
    for kw, rc in ((dict(heads=3), INV), (dict(heads=0), INV), (dict(heads=-2), INV), (dict(heads=65538), INV), (dict(qp=0), INV), (dict(out=0), INV),
                   (dict(qp=FAR + 2), MIS), (dict(out=FAR + 8), MIS), (dict(qa=260), MIS), (dict(ob=4), MIS), (dict(ws=0), INV), (dict(ws=FAKE + 8), MIS),
                   (dict(size=need - 1), INV), (dict(qa=1 << 50), INV), (dict(oa=0), INV), (dict(oa=192), INV), (dict(ob=0), INV), (dict(ob=56), INV),
                   (dict(out=FAR), INV), (dict(out=FAR + 128), INV), (dict(qp=(1 << 64) - 4096), INV),
                   (dict(scores=s(nan, 0.0, 0, None)), INV), (dict(scores=s(inf, 0.0, 0, None)), INV), (dict(scores=s(1.0, -1.0, 0, None)), INV),
                   (dict(scores=s(1.0, nan, 0, None)), INV), (dict(scores=s(1.0, 2e30, 0, None)), INV), (dict(scores=s(1.0, 1e-40, 0, None)), INV),
                   (dict(scores=s(1.0, 0.0, -1, None)), INV), (dict(scores=s(1.0, 0.0, 0, FAKE + 2)), MIS)):
        assert attend(jb, **kw) == rc, kw


def test_bad_appends(jb):
    r = lambda *a: jb.jb_rotation(*a)  # noqa: E731
    assert append(jb, n=0, k=0, v=0, qp=0) == 0
    for kw, rc in ((dict(rot=r(0, 64, 0)), INV), (dict(rot=r(FAKE + 4, 64, 0)), MIS), (dict(rot=r(FAKE, 0, 0)), INV), (dict(rot=r(FAKE, 63, 0)), INV),
                   (dict(rot=r(FAKE, 66, 0)), INV), (dict(rot=r(FAKE, -2, 0)), INV), (dict(heads=-1), INV), (dict(heads=65537), INV), (dict(n=-1), INV),
                   (dict(rows=0), INV), (dict(pos=0), INV), (dict(rows=FAKE + 2), MIS), (dict(turns=FAKE + 2), MIS), (dict(k=0), INV), (dict(v=0), INV),
                   (dict(qp=0), INV), (dict(out=0), INV), (dict(k=FAR + 8), MIS), (dict(v=FAR + 4), MIS), (dict(qp=FAR + 8), MIS), (dict(out=FAR + 4), MIS),
                   (dict(ka=132), MIS), (dict(vb=4), MIS), (dict(qa=260), MIS), (dict(ob=68), MIS), (dict(va=1 << 50), INV), (dict(oa=1 << 50), INV),
                   (dict(k=(1 << 64) - 64), INV), (dict(n=2, oa=192), INV), (dict(ob=56), INV)):
        assert append(jb, **kw) == rc, kw
    L, q, kv = jb.lib(), C.byref(pages(jb)), layer(jb)
    assert L.jb_cache_append(q, None, C.byref(r(FAKE, 64, 0)), None, 0, 0, 0, None, 0, 0, p(FAR), 128, 64, p(FAR), 128, 64, p(FAKE), p(FAKE), None, 1, None) == INV
    assert L.jb_cache_append(q, C.byref(kv), None, None, 0, 0, 0, None, 0, 0, p(FAR), 128, 64, p(FAR), 128, 64, p(FAKE), p(FAKE), None, 1, None) == INV


def test_appends_that_share_bytes(jb):
    """One row of queries, keys and values is 512 elements here: 4 heads of 64, then 2, then 2."""
    row = dict(n=3, qa=512, ka=512, va=512, oa=512, qp=FAR, k=FAR + 512, v=FAR + 768)
    gap = FAR + 3 * 1024
    bad = -3  # a misaligned list ends the calls that share nothing before anything is launched
    def rc(**kw):
        return append(jb, **{**row, **kw})
    # refused: turned queries over keys, values, other queries, the cache; keys in the cache
    for kw in (dict(out=FAR + 512), dict(out=FAR + 768), dict(out=FAR + 128), dict(out=FAR - 128), dict(out=FAR + 1024), dict(out=FAR, oa=256), dict(out=FAR, ob=80, oa=512),
               dict(out=FAKE, oa=256), dict(out=FAKE + (1 << 24)), dict(k=FAKE), dict(v=FAKE + (1 << 24) + 1024), dict(qp=FAKE + 2048, out=gap), dict(out=FAR, qa=256, k=gap, v=gap + 8192)):
        assert rc(**kw) == INV, kw
    assert rc(turns=FAKE + 2) == bad and rc(turns=FAKE + 2, out=FAR) == bad


def q4(jb, codes=FAKE, scale=FAKE + (1 << 30), numel=128 * 256, out=128, inner=256, dtype=1, x=FAR, xs=256, n=2, bias=0, y=FAR + (1 << 20), ys=128, none=False, ws=0, size=0):
    w = jb.jb_q4_segment(codes, scale, numel, 0)
    return jb.lib().jb_q4_matmul(None if none else C.byref(w), out, inner, dtype, p(x), xs, n, p(bias), p(y), ys, p(ws), size, None)


def test_bad_products(jb):
    assert q4(jb, n=0, x=0, y=0, codes=0) == 0
    for kw, rc in ((dict(dtype=2), DTYPE), (dict(none=True), INV), (dict(out=0), INV), (dict(inner=0), INV), (dict(inner=32, numel=128 * 32), INV),
                   (dict(inner=250), INV), (dict(inner=65600, numel=128 * 65600), INV), (dict(n=-1), INV), (dict(numel=128 * 256 - 1), INV), (dict(out=127), INV),
                   (dict(out=(1 << 30) + 1, inner=64, numel=64 * ((1 << 30) + 1), ys=(1 << 30) + 1), INV), (dict(codes=0), INV), (dict(scale=0), INV), (dict(x=0), INV), (dict(y=0), INV), (dict(codes=FAKE + 4), MIS), (dict(scale=FAKE + 2), MIS),
                   (dict(x=FAR + 8), MIS), (dict(xs=260), MIS), (dict(y=FAR + 1), MIS), (dict(bias=FAKE + 1), MIS), (dict(dtype=0, y=FAR + 2), MIS),
                   (dict(xs=1 << 50), INV), (dict(ys=1 << 50), INV), (dict(ys=127), INV), (dict(y=FAR), INV), (dict(y=FAR + 510), INV), (dict(y=FAKE + 100), INV),
                   (dict(y=FAKE + (1 << 30)), INV), (dict(bias=FAR + (1 << 20) + 2), INV), (dict(x=(1 << 64) - 256), INV), (dict(codes=(1 << 64) - 1024), INV)):
        assert q4(jb, **kw) == rc, kw
    need = lambda *a: jb.lib().jb_q4_matmul_workspace(*a)  # noqa: E731
    assert need(128, 256, 1, 2) == 0 and need(4096, 4096, 2, 1) == 0 and need(4096, 4000, 1, 1) == 0 and need(0, 4096, 1, 1) == 0
    assert need((1 << 30) + 1, 64, 1, 1) == 0
    big = dict(numel=4096 * 4096, out=4096, inner=4096, xs=4096, ys=4096, n=9, ws=FAKE, size=need(4096, 4096, 1, 9))
    assert big["size"] > 9 * 4096 * 2
    for kw, rc in ((dict(ws=0), INV), (dict(ws=FAKE + 8), MIS), (dict(size=big["size"] - 1), INV)):
        assert q4(jb, **{**big, **kw}) == rc, kw


def test_python_refuses(jb, monkeypatch):
    import torch
    i32, f32 = torch.int32, torch.float32
    library = Launches()
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    new = lambda *shape, dtype=i32, at=0: on_device(at, torch.zeros(shape, dtype=dtype))[0]  # noqa: E731
    cache = jb.KVCache(jb.PageTable(new(2, 3), new(2), new(6), 16), [new(6, 2, 16, 64, dtype=f32)], [new(6, 2, 16, 64, dtype=f32)])
    cpu = torch.zeros(2, dtype=i32)
    for bad in ((cpu, cpu, cpu), (new(2), new(2), new(5)), (new(2), new(3), new(5, at=1)), (new(2), new(3, at=1), new(5)), (new(2), new(3), new(5, dtype=f32)),
                (new(2), new(3), new(5, 1))):
        with pytest.raises(ValueError):
            jb.DraftTrees(*bad)
    for bad in (torch.zeros(4, dtype=torch.int64), new(4), new(4, 2, dtype=torch.int64), new(8, dtype=torch.int64)[::2]):
        with pytest.raises(ValueError):
            jb.Rotation(bad)
    with pytest.raises(ValueError):
        jb.Rotation.steps_of([1.0, float("inf")])
    with pytest.raises(ValueError):
        jb.Rotation.powers(7)
    rotation, t = jb.Rotation(new(32, dtype=torch.int64)), jb.DraftTrees(new(2), new(3), new(5))
    kv = lambda n, at=0, dtype=f32: new(n, 2, 64, dtype=dtype, at=at)  # noqa: E731
    q = lambda n, at=0, dtype=f32: new(n, 4, 64, dtype=dtype, at=at)  # noqa: E731
    good = dict(q=q(5), k=kv(5), v=kv(5), rows=new(5), pos=new(5), rotation=rotation, turns=new(5), q_out=q(5))
    calls = []
    for change in (dict(q=q(5, 1)), dict(k=kv(5, 1)), dict(v=kv(4)), dict(rows=new(4)), dict(pos=new(5, at=1)), dict(turns=new(4)), dict(turns=new(5, at=1)),
                   dict(q_out=q(5, dtype=torch.bfloat16)), dict(q=None), dict(q=new(5, 4, 32, dtype=f32)), dict(rotation=jb.Rotation(new(32, dtype=torch.int64, at=1)))):
        calls.append(("jb_cache_append", (cache, 0), {**good, **change}))
    good = dict(q=q(5), trees=t, out=q(5), slopes=new(4, dtype=f32), workspace=new(1 << 20))
    for change in (dict(q=q(4)), dict(q=q(5, 1)), dict(out=q(5, 1)), dict(trees=jb.DraftTrees(new(2, at=1), new(3, at=1), new(5, at=1))), dict(slopes=new(3, dtype=f32)),
                   dict(slopes=new(4, dtype=f32, at=1)), dict(workspace=new(1 << 20, at=1))):
        calls.append(("jb_attend_tree", (cache, 0), {**good, **change}))
    good = dict(trees=t, leaves=new(2), status=new(1))
    for change in (dict(leaves=new(3)), dict(leaves=new(2, at=1)), dict(status=new(2)), dict(status=new(1, at=1)),
                   dict(trees=jb.DraftTrees(new(2, at=1), new(3, at=1), new(5, at=1)))):
        calls.append(("jb_cache_keep", (cache,), {**good, **change}))
    table = jb.Q4Table([(new(128 * 32, dtype=torch.uint8), new(128, dtype=f32), 128 * 64)])
    good = dict(x=new(3, 64, dtype=f32), out_features=128, bias=new(128, dtype=f32), out=new(3, 128, dtype=f32))
    for change in (dict(x=new(3, 64, dtype=f32, at=1)), dict(x=torch.zeros(3, 64)), dict(x=new(64, dtype=f32)), dict(x=new(64, 3, dtype=f32).T), dict(bias=new(64, dtype=f32)),
                   dict(bias=new(128, dtype=torch.bfloat16)), dict(out=new(3, 127, dtype=f32)), dict(out=new(128, 3, dtype=f32).T), dict(out=new(3, 128, dtype=f32, at=1)), dict(workspace=new(64, at=1))):
        calls.append(("jb_q4_matmul", (table, 0), {**good, **change}))
    elsewhere = jb.Q4Table([(new(128 * 32, dtype=torch.uint8, at=1), new(128, dtype=f32), 128 * 64)])
    calls.append(("jb_q4_matmul", (elsewhere, 0), good))
    monkeypatch.setattr(jb, "lib", lambda: library)
    for name, first, kw in calls:
        with pytest.raises(ValueError):
            getattr(jb, name)(*first, **kw, stream=1)
    with pytest.raises(TypeError):
        jb.jb_q4_matmul(table, 0, new(3, 64, dtype=torch.float16), 128, stream=1)
    with pytest.raises(IndexError):
        jb.jb_q4_matmul(table, 1, new(3, 64, dtype=f32), 128, stream=1)
    for current in (1,):
        monkeypatch.setattr(torch.cuda, "current_device", lambda: current)
        with pytest.raises(ValueError, match="device"):
            jb.jb_attend_tree(cache, 0, q(5), t, out=q(5), workspace=new(1 << 20), stream=1)
        with pytest.raises(ValueError, match="device"):
            jb.jb_q4_matmul(table, 0, new(3, 64, dtype=f32), 128, out=new(3, 128, dtype=f32), stream=1)
    assert library.calls == 0


def test_steps_are_the_frequencies(jb):
    f = np.array([1.0, 0.25, 1e-5, 2 * np.pi / 3, 0.0, -1.0])
    turns = jb.Rotation.steps_of(f).view(np.uint64).astype(np.float64) / 2.0**64
    want = np.mod(f / (2 * np.pi), 1.0)
    assert np.abs(turns - want).max() <= 2.0**-53


def test_sizes_of_workspaces_do_not_pile_up(jb):
    """A server's numbers of rows are many; what is remembered of them is not."""
    import torch
    new = lambda *shape, dtype: on_device(0, torch.zeros(shape, dtype=dtype))[0]  # noqa: E731
    table = jb.Q4Table([(new(128 * 32, dtype=torch.uint8), new(128, dtype=torch.float32), 128 * 64)])
    want = [int(jb.lib().jb_q4_matmul_workspace(4096, 4096, 1, n)) for n in range(1, 3000)]
    assert [table.matmul_workspace(4096, 4096, torch.bfloat16, n) for n in range(1, 3000)] == want and max(want) > 0
    assert len(table._matmul_bytes) <= 1024
    assert table.matmul_workspace(4096, 4096, torch.bfloat16, 9) == want[8]


@pytest.mark.parametrize("out,inner,rows_bf16,rows_f32", [(5120, 20480, 1, 1), (4096, 16384, 2, 1), (20480, 5120, 7, 4), (4096, 4096, 9, 5), (1024, 4096, 9, 5),
                                                          (2048, 2048, 16, 8), (16384, 1024, 17, 9), (4096, 1024, 24, 12), (1024, 1024, 32, 16),
                                                          (8192, 8192, 4, 2), (512, 512, 1 << 20, 1 << 20)])
def test_from_how_many_rows_on_products_are_cut_into_tiles(jb, out, inner, rows_bf16, rows_f32):
    """Where the kernels' measured times cross, on a GB300; the tiles alone work in a workspace."""
    need = lambda dtype, n: jb.lib().jb_q4_matmul_workspace(out, inner, dtype, n)  # noqa: E731
    for dtype, first in ((1, rows_bf16), (0, rows_f32)):
        rows = [n for n in list(range(1, 70)) + [1000, 100_000] if need(dtype, n) > 0]
        assert rows == [n for n in list(range(1, 70)) + [1000, 100_000] if n >= first], (dtype, rows[:1])


def test_products_of_more_rows_than_2_to_the_30(jb):
    """Passes over the rows count them in 31 bits, beyond the last of which there is no room."""
    most = 1 << 30
    for dtype in (0, 1):
        for n in (most + 1, (1 << 31) - 1):
            assert q4(jb, n=n, dtype=dtype, xs=0, out=1, numel=256, ys=1) == INV
            assert jb.lib().jb_q4_matmul_workspace(4096, 4096, dtype, n) == 0
        assert q4(jb, n=most, dtype=dtype, xs=0, out=1, numel=256, ys=1, bias=FAKE + 1) == MIS   # a misaligned bias ends it, not its rows
        assert jb.lib().jb_q4_matmul_workspace(4096, 4096, dtype, most) > 0
