"""Host threads that call at the same time: a call is several launches over one workspace and one page table, so the next one's
may not come between them. The library is a stand-in that stays in each call for a moment."""
import threading
import time

import pytest

from test_answer_host import jb, on_device  # noqa: F401  (a fixture)


class Slow:
    """A library whose calls take a while, and that says how many were in it at a time."""

    def __init__(self):
        self.inside, self.most, self.calls, self.own = 0, 0, 0, threading.Lock()

    def __getattr__(self, name):
        def call(*args):
            if name.endswith("_workspace"):
                return 4096
            with self.own:
                self.inside += 1
                self.calls += 1
                self.most = max(self.most, self.inside)
            time.sleep(2e-3)
            with self.own:
                self.inside -= 1
            return 0
        return call


def calls_of(jb):  # noqa: F811
    """Groups of calls that work on the same objects, and a call on others."""
    import torch
    i32, f32 = torch.int32, torch.float32
    new = lambda *shape, dtype=i32: on_device(0, torch.zeros(shape, dtype=dtype))[0]  # noqa: E731
    pages = jb.PageTable(new(2, 3), new(2), new(6), 16)
    kv = lambda: [new(6, 2, 16, 64, dtype=f32)]  # noqa: E731
    cache, twin = jb.KVCache(pages, kv(), kv()), jb.KVCache(pages, kv(), kv())
    trees, rotation = jb.DraftTrees(new(2), new(3), new(5)), jb.Rotation(new(32, dtype=torch.int64))
    q, k, st = new(5, 4, 64, dtype=f32), new(5, 2, 64, dtype=f32), dict(status=new(1), stream=1)
    table, other = (jb.Q4Table([(new(128 * 32, dtype=torch.uint8), new(128, dtype=f32), 128 * 64)]) for _ in range(2))
    x, y = new(3, 64, dtype=f32), new(3, 128, dtype=f32)
    of_cache = [lambda c=c, f=f: f(c) for c in (cache, twin) for f in (
        lambda c: jb.jb_attend_tree(c, 0, q, trees, out=q.clone(), stream=1), lambda c: jb.jb_cache_keep(c, trees, new(2), **st),
        lambda c: jb.jb_cache_append(c, 0, q, k, k, new(5), new(5), rotation, q_out=q, stream=1), lambda c: jb.jb_cache_reserve(c, new(2), new(2), **st),
        lambda c: jb.jb_cache_free(c, new(2), stream=1), lambda c: jb.jb_cache_fork(c, new(1), new(1), **st), lambda c: jb.jb_cache_compact(c, **st),
        lambda c: jb.jb_cache_write(c, 0, k, k, new(5), new(5), stream=1), lambda c: jb.jb_attend(c, 0, q, new(5), new(5), out=q.clone(), stream=1))]
    of_table = [lambda: jb.jb_q4_matmul(table, 0, x, 128, out=y, stream=1), lambda: jb.jb_perturb_q4(table, (1, 2, 3), 0.1, stream=1)]
    return of_cache, of_table, lambda: jb.jb_q4_matmul(other, 0, x, 128, out=y.clone(), stream=1)


def all_at_once(calls):
    failed = []
    def run(call):
        try:
            for _ in range(3):
                call()
        except Exception as e:  # noqa: BLE001
            failed.append(e)
    threads = [threading.Thread(target=run, args=(c,)) for c in calls]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not failed, failed[0]


@pytest.fixture
def slow(jb, monkeypatch):  # noqa: F811
    import torch
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: False)
    jb._need_torch()
    monkeypatch.setattr(jb, "_new", lambda stream, make, *args, **kw: make(*args, **kw))
    groups = calls_of(jb)
    library = Slow()
    monkeypatch.setattr(jb, "lib", lambda: library)
    return library, groups


def test_calls_on_one_page_table_follow_one_another(slow):
    library, (calls, _, _) = slow
    all_at_once(calls)
    assert library.calls == 3 * len(calls) and library.most == 1


def test_products_with_one_table_follow_one_another(slow):
    library, (_, calls, _) = slow
    all_at_once(2 * calls)
    assert library.calls == 3 * 2 * len(calls) and library.most == 1


def test_calls_on_other_objects_do_not_wait(slow):
    library, (of_cache, of_table, other) = slow
    all_at_once([of_cache[0], of_table[0], other])
    assert library.most > 1


def test_a_call_that_fails_leaves_the_others_free(slow, jb):  # noqa: F811
    library, (of_cache, of_table, _) = slow
    library.jb_status_string = lambda rc: b"failed"
    library.__dict__["jb_attend_tree"] = library.__dict__["jb_q4_matmul"] = lambda *args: -1
    for call in (of_cache[0], of_table[0]):
        with pytest.raises(RuntimeError):
            call()
    all_at_once([of_cache[1], of_table[1]])
    assert library.calls == 6


def test_a_finalizer_may_call_while_its_thread_is_in_a_call(slow, jb, monkeypatch):  # noqa: F811
    """The collector runs where memory is asked for, and with it whatever frees the rows of an answer that nobody holds."""
    library, (of_cache, of_table, _) = slow
    seen = []

    def new(stream, make, *args, **kw):
        if not seen and make is not __import__("torch").cuda.is_current_stream_capturing:
            seen.append(1)
            of_cache[4]()                                                 # jb_cache_free, of the same pages
        return make(*args, **kw)
    monkeypatch.setattr(jb, "_new", new)
    t = threading.Thread(target=of_cache[0], daemon=True)                 # jb_attend_tree, which makes its workspace
    t.start()
    t.join(10)
    assert not t.is_alive() and seen and library.calls == 2
