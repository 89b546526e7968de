"""What the calls that write answers refuse, before anything touches CUDA. The device addresses here are
never dereferenced: every call returns an error or is a no-op."""
import ctypes as C

import pytest

INV, DTYPE, MIS = -1, -2, -3
FAKE = 0x7F0000000000


@pytest.fixture(scope="module")
def jb():
    from paper_2306_10015_gb300 import build
    build.build()
    import paper_2306_10015_gb300 as pkg
    pkg.lib()
    return pkg


def p(x):
    return C.c_void_p(x)


def pages(jb, **kw):
    v = dict(table=FAKE, lens=FAKE + 4096, refs=FAKE + 8192, n_rows=4, row_pages=8, n_pages=32, page_tokens=16)
    v.update(kw)
    return jb.jb_pages(*v.values())


def layer(jb, **kw):
    v = dict(k=FAKE, v=FAKE + (1 << 24), page_stride=2 * 64 * 16, heads=2, head_dim=64, dtype=1, by_token=0)
    v.update(kw)
    return jb.jb_kv(*v.values())


BAD_PAGES = [(dict(table=0), INV), (dict(lens=0), INV), (dict(refs=0), INV), (dict(n_rows=0), INV), (dict(n_rows=65537), INV),
             (dict(row_pages=0), INV), (dict(n_pages=0), INV), (dict(n_pages=(1 << 30) + 1), INV), (dict(page_tokens=0), INV),
             (dict(page_tokens=8), INV), (dict(page_tokens=24), INV), (dict(page_tokens=1040), INV),
             (dict(row_pages=1 << 27), INV), (dict(table=FAKE + 2), MIS), (dict(lens=FAKE + 1), MIS), (dict(refs=FAKE + 3), MIS)]
BAD_LAYERS = [(dict(k=0), INV), (dict(v=0), INV), (dict(heads=0), INV), (dict(head_dim=0), INV), (dict(head_dim=264), INV),
              (dict(dtype=2), DTYPE), (dict(head_dim=60), MIS), (dict(dtype=0, head_dim=62), MIS), (dict(k=FAKE + 8), MIS),
              (dict(v=FAKE + 2), MIS), (dict(page_stride=2 * 64 * 16 - 8), INV), (dict(page_stride=2 * 64 * 16 + 4), MIS),
              (dict(page_stride=1 << 60), INV), (dict(k=(1 << 64) - 4096), INV)]


def test_bad_page_tables(jb):
    L = jb.lib()
    for kw, rc in BAD_PAGES:
        q, kv = C.byref(pages(jb, **kw)), layer(jb)
        assert L.jb_cache_reserve(q, p(FAKE), p(FAKE), 1, p(FAKE), None) == rc, kw
        assert L.jb_cache_free(q, p(FAKE), 1, None) == rc, kw
        assert L.jb_cache_fork(q, C.byref(kv), 1, p(FAKE), p(FAKE), 1, p(FAKE), p(FAKE), 1 << 20, None) == rc, kw
        assert L.jb_cache_compact(q, C.byref(kv), 1, p(FAKE), p(FAKE), 1 << 20, None) == rc, kw
        assert L.jb_cache_write(q, C.byref(kv), p(FAKE), 128, 64, p(FAKE), 128, 64, p(FAKE), p(FAKE), 1, None) == rc, kw
        assert attend(jb, q, kv) == rc, kw
        assert L.jb_cache_workspace(q, 1) == 0
    assert L.jb_cache_reserve(None, p(FAKE), p(FAKE), 1, p(FAKE), None) == INV


def attend(jb, q, kv, scores=None, qp=FAKE, qa=256, qb=64, heads=4, rows=FAKE, pos=FAKE, n=1, out=FAKE, oa=256, ob=64, ws=FAKE, size=None):
    s = jb.jb_scores(0.125, 0.0, 0, None) if scores is None else scores
    size = 1 << 40 if size is None else size
    return jb.lib().jb_attend(q, C.byref(kv), C.byref(s), p(qp), qa, qb, heads, p(rows), p(pos), n, p(out), oa, ob, p(ws), size, None)


def test_bad_layers(jb):
    L, q = jb.lib(), C.byref(pages(jb))
    for kw, rc in BAD_LAYERS:
        kv = layer(jb, **kw)
        assert L.jb_cache_fork(q, C.byref(kv), 1, p(FAKE), p(FAKE), 1, p(FAKE), p(FAKE), 1 << 20, None) == rc, kw
        assert L.jb_cache_compact(q, C.byref(kv), 1, p(FAKE), p(FAKE), 1 << 20, None) == rc, kw
        assert L.jb_cache_write(q, C.byref(kv), p(FAKE), 128, 64, p(FAKE), 128, 64, p(FAKE), p(FAKE), 1, None) == rc, kw
        assert attend(jb, q, kv) == rc, kw
    two = (jb.jb_kv * 2)(layer(jb), layer(jb, heads=1))                 # layers of unlike geometry
    assert L.jb_cache_compact(q, two, 2, p(FAKE), p(FAKE), 1 << 20, None) == INV
    assert L.jb_cache_compact(q, two, 0, p(FAKE), p(FAKE), 1 << 20, None) == INV
    assert L.jb_cache_compact(q, None, 1, p(FAKE), p(FAKE), 1 << 20, None) == INV


def test_bad_lists_and_workspaces(jb):
    L, q, kv = jb.lib(), C.byref(pages(jb)), layer(jb)
    for n, a, b, rc in ((-1, FAKE, FAKE, INV), (16385, FAKE, FAKE, INV), (1, 0, FAKE, INV), (1, FAKE, 0, INV), (1, FAKE + 2, FAKE, MIS)):
        assert L.jb_cache_reserve(q, p(a), p(b), n, p(FAKE), None) == rc
        assert L.jb_cache_fork(q, C.byref(kv), 1, p(a), p(b), n, p(FAKE), p(FAKE), 1 << 30, None) == rc
    assert L.jb_cache_reserve(q, p(FAKE), p(FAKE), 1, None, None) == INV
    assert L.jb_cache_reserve(q, p(FAKE), p(FAKE), 1, p(FAKE + 2), None) == MIS
    assert L.jb_cache_free(q, None, 1, None) == INV and L.jb_cache_free(q, p(FAKE), -1, None) == INV
    assert L.jb_cache_free(q, None, 0, None) == 0
    need = L.jb_cache_workspace(q, 3)
    assert need >= 4 * 3 * 8                                             # the parents' rows at least
    fork = lambda ws, size: L.jb_cache_fork(q, C.byref(kv), 1, p(FAKE), p(FAKE), 3, p(FAKE), p(ws), size, None)  # noqa: E731
    assert fork(0, need) == INV and fork(FAKE, need - 1) == INV and fork(FAKE + 8, need) == MIS
    need = L.jb_cache_workspace(q, 0)
    compact = lambda ws, size: L.jb_cache_compact(q, C.byref(kv), 1, None, p(ws), size, None)  # noqa: E731
    assert compact(0, need) == INV and compact(FAKE, need - 1) == INV and compact(FAKE + 4, need) == MIS
    assert L.jb_cache_workspace(q, -1) == 0 and L.jb_cache_workspace(None, 1) == 0


def test_bad_writes(jb):
    L, q, kv = jb.lib(), C.byref(pages(jb)), layer(jb)
    w = lambda k=FAKE, a=128, b=64, v=FAKE, c=128, d=64, rows=FAKE, pos=FAKE, n=1: L.jb_cache_write(  # noqa: E731
        q, C.byref(kv), p(k), a, b, p(v), c, d, p(rows), p(pos), n, None)
    assert w(n=0, k=0) == 0 and w(n=-1) == INV and w(k=0) == INV and w(v=0) == INV and w(rows=0) == INV
    assert w(k=FAKE + 8) == MIS and w(v=FAKE + 4) == MIS and w(a=132) == MIS and w(d=4) == MIS and w(c=1 << 50) == INV
    assert L.jb_cache_write(q, None, p(FAKE), 128, 64, p(FAKE), 128, 64, p(FAKE), p(FAKE), 1, None) == INV


def test_bad_attention(jb):
    q, kv = C.byref(pages(jb)), layer(jb)
    s = lambda *a: jb.jb_scores(*a)  # noqa: E731
    inf, nan = float("inf"), float("nan")
    assert attend(jb, q, kv, n=0, qp=0) == 0
    for kw, rc in ((dict(heads=3), INV), (dict(heads=0), INV), (dict(heads=-2), INV), (dict(n=-1), INV), (dict(qp=0), INV), (dict(out=0), INV),
                   (dict(rows=0), INV), (dict(pos=0), INV), (dict(qp=FAKE + 2), MIS), (dict(out=FAKE + 8), MIS), (dict(qa=260), MIS), (dict(ob=4), MIS),
                   (dict(ws=0), INV), (dict(ws=FAKE + 8), MIS), (dict(size=16), INV), (dict(qa=1 << 50), INV),
                   (dict(scores=s(nan, 0.0, 0, None)), INV), (dict(scores=s(inf, 0.0, 0, None)), INV), (dict(scores=s(1.0, -1.0, 0, None)), INV),
                   (dict(scores=s(1.0, nan, 0, None)), INV), (dict(scores=s(1.0, 2e30, 0, None)), INV), (dict(scores=s(1.0, 1e-40, 0, None)), INV), (dict(scores=s(1.0, 0.0, -1, None)), INV), (dict(scores=s(1.0, 0.0, 0, FAKE + 2)), MIS)):
        assert attend(jb, q, kv, **kw) == rc, kw
    assert jb.lib().jb_attend(q, None, C.byref(s(1.0, 0.0, 0, None)), p(FAKE), 256, 64, 4, p(FAKE), p(FAKE), 1, p(FAKE), 256, 64, p(FAKE), 1 << 40, None) == INV
    assert jb.lib().jb_attend_workspace(None, 4) == 0 and jb.lib().jb_attend_workspace(C.byref(kv), 1) == 0


def test_bad_sampling(jb):
    L = jb.lib()
    def sample(logits=FAKE, stride=100, dtype=0, n=2, vocab=100, words=FAKE, tokens=FAKE, lp=FAKE, t=None, settings=True):
        s = jb.jb_sampling(t, None, None, None)
        return L.jb_sample(p(logits), stride, dtype, n, vocab, C.byref(s) if settings else None, p(words), p(tokens), p(lp), None)
    assert sample(n=0, logits=0) == 0
    for kw, rc in ((dict(dtype=2), DTYPE), (dict(n=-1), INV), (dict(vocab=0), INV), (dict(vocab=262145), INV), (dict(settings=False), INV),
                   (dict(logits=0), INV), (dict(words=0), INV), (dict(tokens=0), INV), (dict(logits=FAKE + 2), MIS), (dict(logits=FAKE + 1, dtype=1), MIS),
                   (dict(words=FAKE + 2), MIS), (dict(tokens=FAKE + 1), MIS), (dict(lp=FAKE + 2), MIS), (dict(t=FAKE + 2), MIS), (dict(stride=1 << 50), INV)):
        assert sample(**kw) == rc, kw


def test_python_refuses_tensors_that_are_not_on_the_gpu(jb):
    import torch
    z = torch.zeros(4, dtype=torch.int32)
    with pytest.raises(ValueError):
        jb.PageTable(torch.zeros(4, 8, dtype=torch.int32), z, z, 16)
    with pytest.raises(ValueError):
        jb.jb_sample(torch.zeros(4, 10), z)
    with pytest.raises(ValueError):
        jb.jb_cache_free(None, z)
    with pytest.raises(ValueError):
        jb.jb_cache_reserve(None, z, z)


def test_outputs_that_overlap_are_refused(jb):
    q, kv = C.byref(pages(jb)), layer(jb)
    for kw in (dict(n=2, oa=0), dict(n=2, oa=56), dict(ob=0), dict(ob=56, oa=64)):
        assert attend(jb, q, kv, **kw) == INV, kw


def test_outputs_that_share_bytes_are_refused_in_any_order(jb):
    """Every small pair of strides against the places that the outputs take. A workspace off its grid ends the calls
    whose outputs are apart before anything is launched."""
    q, kv = C.byref(pages(jb)), layer(jb, head_dim=8, page_stride=2 * 8 * 16)
    apart = 0
    for n in (1, 2, 3, 5):
        for heads in (2, 4, 6):
            for oa in range(0, 88, 8):
                for ob in range(0, 88, 8):
                    places = [i * oa + h * ob + e for i in range(n) for h in range(heads) for e in range(8)]
                    rc = MIS if len(set(places)) == len(places) else INV
                    apart += rc == MIS
                    assert attend(jb, q, kv, n=n, heads=heads, oa=oa, ob=ob, ws=FAKE + 8) == rc, (n, heads, oa, ob)
    assert apart > 400


def test_outputs_of_long_strides(jb):
    q, kv, far = C.byref(pages(jb)), layer(jb, head_dim=8, page_stride=2 * 8 * 16), 1 << 48
    for n, heads, oa, ob, rc in ((2, 65536, far, 8, MIS), (2, 65536, 65536 * 8, 8, MIS), (2, 65536, 65535 * 8, 8, INV), (2147483647, 65536, far, far, INV),
                                 (2147483647, 2, 8, far, MIS), (2147483647, 65536, far - 8, far, MIS), (3, 65536, far, far - 8, MIS),
                                 (2147483647, 2, 8, 8 * 2147483647, MIS), (2147483647, 2, 8, 8 * 2147483646, INV)):
        assert attend(jb, q, kv, n=n, heads=heads, oa=oa, ob=ob, ws=FAKE + 8) == rc, (n, heads, oa, ob)


def on_device(index, *tensors):
    """The tensors as if they were on that CUDA device."""
    import torch

    class There(torch.Tensor):
        where = index
        is_cuda = property(lambda self: True)

        def get_device(self):
            return self.where

    return [t.as_subclass(There) for t in tensors]


class Launches:
    """A library that counts its calls."""

    def __init__(self):
        self.calls = 0

    def __getattr__(self, name):
        def call(*args):
            self.calls += 1
            return 0
        return call


def a_call(jb, name, lists, cache_on):
    """The call's arguments; `lists` maps an argument's place to its device, 0 by default."""
    import torch
    i32, f32 = torch.int32, torch.float32
    table, lens, refs = on_device(cache_on, torch.zeros(2, 3, dtype=i32), torch.zeros(2, dtype=i32), torch.zeros(6, dtype=i32))
    k, v = on_device(cache_on, torch.zeros(6, 2, 16, 64), torch.zeros(6, 2, 16, 64))
    cache = jb.KVCache(jb.PageTable(table, lens, refs, 16), [k], [v])
    new = lambda *shape, dtype=i32: torch.zeros(shape, dtype=dtype)  # noqa: E731
    args = dict(jb_cache_reserve=dict(rows=new(2), tokens=new(2), status=new(1)), jb_cache_free=dict(rows=new(2)),
                jb_cache_fork=dict(parents=new(2), children=new(2), status=new(1)), jb_cache_compact=dict(status=new(1)),
                jb_cache_write=dict(k=new(2, 2, 64, dtype=f32), v=new(2, 2, 64, dtype=f32), rows=new(2), pos=new(2)),
                jb_attend=dict(q=new(2, 4, 64, dtype=f32), rows=new(2), pos=new(2), out=new(2, 4, 64, dtype=f32), slopes=new(4, dtype=f32),
                               workspace=new(1 << 20)),
                jb_sample=dict(logits=new(2, 9, dtype=f32), words=new(2), temperature=new(2, dtype=f32), top_k=new(2), top_p=new(2, dtype=f32),
                               min_p=new(2, dtype=f32), tokens=new(2), logprobs=new(2, dtype=f32)))[name]
    args = {a: on_device(lists.get(a, lists.get("all", 0)), t)[0] for a, t in args.items()}
    first = {"jb_sample": (), "jb_attend": (cache, 0), "jb_cache_write": (cache, 0)}.get(name, (cache,))
    return first, args


CALLS = dict(jb_cache_reserve=3, jb_cache_free=1, jb_cache_fork=3, jb_cache_compact=1, jb_cache_write=4, jb_attend=6, jb_sample=8)


@pytest.mark.parametrize("name", CALLS)
def test_tensors_of_another_device_are_refused(jb, name, monkeypatch):
    import torch
    current = [0]
    library = Launches()
    monkeypatch.setattr(torch.cuda, "current_device", lambda: current[0])
    _, args = a_call(jb, name, {}, 0)
    assert len(args) == CALLS[name]
    for one in args:                                                     # one argument elsewhere
        first, args = a_call(jb, name, {one: 1}, 0)
        with monkeypatch.context() as m:
            m.setattr(jb, "lib", lambda: library)
            with pytest.raises(ValueError, match="device"):
                getattr(jb, name)(*first, **args, stream=1)
    for current[0], lists, cache_on in ((0, 1, 1), (1, 0, 0), (0, 1, 0), (1, 1, 0)):
        if name == "jb_sample" and current[0] == lists:
            continue                                                     # it has no cache
        first, args = a_call(jb, name, {"all": lists}, cache_on)
        with monkeypatch.context() as m:
            m.setattr(jb, "lib", lambda: library)
            with pytest.raises(ValueError, match="device"):
                getattr(jb, name)(*first, **args, stream=1)
    assert library.calls == 0


@pytest.mark.parametrize("name", ["jb_cache_reserve", "jb_cache_free", "jb_cache_write", "jb_attend", "jb_sample"])
@pytest.mark.parametrize("device", [0, 3])
def test_tensors_of_the_current_device_are_taken(jb, name, device, monkeypatch):
    import torch
    library = Launches()
    first, args = a_call(jb, name, {"all": device}, device)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: device)
    monkeypatch.setattr(jb, "lib", lambda: library)
    getattr(jb, name)(*first, **args, stream=1)
    assert library.calls == 1


def test_a_cache_is_on_one_device(jb):
    import torch
    i32 = torch.int32
    whole = lambda a, b, c: jb.PageTable(*on_device(a, torch.zeros(2, 3, dtype=i32)), *on_device(b, torch.zeros(2, dtype=i32)),  # noqa: E731
                                         *on_device(c, torch.zeros(6, dtype=i32)), 16)
    for where in ((0, 0, 1), (0, 1, 0), (1, 0, 0)):
        with pytest.raises(ValueError, match="device"):
            whole(*where)
    kv = lambda at: on_device(at, torch.zeros(6, 2, 16, 64))  # noqa: E731
    for where in ((0, 1), (1, 0), (1, 1)):
        with pytest.raises(ValueError, match="device"):
            jb.KVCache(whole(0, 0, 0), kv(where[0]), kv(where[1]))


def test_the_text_of_a_misaligned_argument_tells_of_segments(jb):
    text = jb.jb_status_string(MIS)
    assert "segment pointer not aligned to its element size" in text and "stride" in text
