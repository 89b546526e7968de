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
