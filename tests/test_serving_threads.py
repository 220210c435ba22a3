"""Calls of several host threads on one stream: the kernels of a call are not mixed with another call's."""
import threading
import time
import types

import numpy as np
import pytest
import torch

import cache8_ref as ref
from paper_2608_12703_gb300 import serving


class Library:
    """Entries that give way to other threads in the middle, as two launches of one call do, and see who else is under way."""

    def __init__(self):
        self.inside, self.met, self.calls = {}, [], 0

    def __getattr__(self, name):
        def entry(*args):
            stream = args[-1]
            self.met.append(self.inside.get(stream, 0))
            self.inside[stream] = self.inside.get(stream, 0) + 1
            time.sleep(0.002)
            self.inside[stream] -= 1
            self.calls += 1
            return 0
        return entry


def made(kind, lib, **kw):
    x = object.__new__(kind)
    x.device, x._index, x._ws, x._lock, x._ref, x._lib = torch.device("cpu"), 0, {}, threading.Lock(), None, lib
    for name, value in kw.items():
        setattr(x, name, value)
    return x


@pytest.fixture
def host(monkeypatch):
    """The classes without a device; each thread's stream is its own attribute."""
    here = threading.local()
    monkeypatch.setattr(serving, "_capturing", lambda: False)
    monkeypatch.setattr(serving, "_current_device", lambda: 0)
    monkeypatch.setattr(serving, "_raw_stream", lambda device: here.stream)
    return here


def callers(lib):
    """A pool's calls and those over the pages that it deals with."""
    i32, A = lambda *x: torch.zeros(x, dtype=torch.int32), serving.A
    pool = made(serving.PagePool, lib, batch=2, n_pages=4, max_pages=2, page_size=16, page_table=i32(2, 2), held=i32(2), refs=i32(4),
                _layout=A.AsrPagePool(), _layouts={}, _bytes=64, _plan=torch.zeros(16, dtype=torch.uint8), _n=1, _reserve=lib.reserve,
                _fork=lib.fork, _compact=lib.compact)
    n, q = i32(2), torch.zeros(2, 1, 2, 64)
    rows = lambda self, *a: A.AsrPagedRows()
    ws = types.SimpleNamespace(asr_spec_paged_attend_ws=lambda *a: 64, asr_spec_paged8_attend_ws=lambda *a: 64)
    cache = made(type("Cache", (serving.PagedCache,), {"_rows": rows, "_weigh_layout": lambda *a: (A.AsrPagedRows(), A.AsrPagedScores(), (1, 1)),
                                                       "_evict_layout": lambda *a: (A.AsrPagedScores(), 64)}), ws, dtype=torch.float32,
                 _attend_layouts={}, _weigh_layouts={}, _evict_layouts={}, _attend=lib.attend, _weigh=lib.weigh, _evict=lib.evict)
    cache8 = made(type("Cache8", (serving.PagedCache8,), {"_rows": rows}), ws, _attend_layouts={}, _append_layouts={}, _attend=lib.attend8,
                  _append=lib.append8, batch=2, kv_heads=2, head_dim=64, _read_only=False)
    score, pos = torch.zeros(2, 2, 4), i32(2, 2, 4)
    return [lambda: pool.reserve(n, n), lambda: pool.fork(n), lambda: pool.compact(), lambda: cache.attend(q, n),
            lambda: cache.weigh(q, score, n, score), lambda: cache.evict(n, score, pos, n, budget=1),
            lambda: cache8.attend(q.half(), n), lambda: cache8.append(q, q, n)]


def run(threads):
    errors = []

    def guarded(f):
        try:
            f()
        except BaseException as e:      # shown in the test's thread
            errors.append(e)
    threads = [threading.Thread(target=guarded, args=(f,)) for f in threads]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    if errors:
        raise errors[0]


def test_calls_on_one_stream_follow_one_another(host):
    lib = Library()
    calls = callers(lib)

    def work(first):
        host.stream = 7
        for i in range(2 * len(calls)):
            calls[(first + i) % len(calls)]()
    run([lambda i=i: work(i) for i in range(4)])
    assert lib.calls == 8 * len(calls) and max(lib.met) == 0


def test_calls_on_their_own_streams_do_not_wait(host):
    lib, meet, met = Library(), threading.Barrier(2, timeout=20), []

    def work(stream):
        host.stream = stream
        calls[0]()

    def both(*args):      # goes on when a call on the other stream is under way too
        met.append(meet.wait())
        return 0
    lib.reserve = both
    calls = callers(lib)
    run([lambda: work(1), lambda: work(2)])
    assert len(met) == 2


@pytest.mark.gpu
def test_two_threads_and_one_pool(built_lib, cuda):
    """Forks and reserves of the same state by two threads on the same stream, each to outputs of its own."""
    from test_gpu_pool import State, i32, samples
    s = State(60, [samples(6, 3000, 16), samples(5, 40, 16), ([700, 0, 90], 0)], 16, 300, 600, layers=2)
    n, page = len(s.lens), s.page
    rng = np.random.default_rng(61)
    forks = [[int(x) for x in rng.integers(-1, n, n)] for _ in range(40)]
    wants = [ref.fork(s.table, s.held, s.refs, p, None, page) for p in forks]
    rows = [[int(x) for x in rng.integers(0, 30, n)] for _ in range(40)]
    reserves = [ref.reserve(s.table, s.held, s.refs, s.lens, r, page) for r in rows]
    parents, needs, lens = [i32(p) for p in forks], [i32(r) for r in rows], i32(s.lens)
    stream = torch.cuda.Stream()
    torch.cuda.synchronize()
    got = {}

    def work(t):
        with torch.cuda.stream(stream):
            for i in range(t, 40, 2):
                got["fork", i] = s.pool.fork(parents[i], **s.outs(False))
                got["reserve", i] = s.pool.reserve(lens, needs[i], **s.outs(False))
    run([lambda: work(0), lambda: work(1)])
    torch.cuda.synchronize()
    assert s.pool.status() == 0
    for i in range(40):
        table, held, refs = got["fork", i]
        assert held.tolist() == wants[i][1].tolist() and refs.tolist() == wants[i][2].tolist()
        s.check_table(table, wants[i][0], wants[i][1], False)
        table, held, refs, counts = got["reserve", i]
        wt, wh, wr, wc, _ = reserves[i]
        assert held.tolist() == wh.tolist() and refs.tolist() == wr.tolist() and counts.tolist() == list(wc)
        s.check_table(table, wt, wh, False)


@pytest.mark.gpu
def test_two_threads_fork_in_place(built_lib, cuda):
    """Two sequences' halves of one state change places over and over, by two threads, in place: any order of whole calls has the
    same counts, and every row is one that a fork can leave."""
    from test_gpu_pool import State, i32
    s = State(62, [([4000, 3000], 0), ([100, 2000], 0)], 16, 300, 3, layers=1, kv_heads=1)
    swap = [i32([1, 0, 2, 3]), i32([0, 1, 3, 2])]
    stream = torch.cuda.Stream()
    torch.cuda.synchronize()

    def work(t):
        with torch.cuda.stream(stream):
            for _ in range(101):
                s.pool.fork(swap[t])
    run([lambda: work(0), lambda: work(1)])
    torch.cuda.synchronize()
    assert s.pool.status() == 0
    table, held, refs = s.table, s.held, s.refs
    for p in ([1, 0, 2, 3], [0, 1, 3, 2]):      # odd numbers of both, which come out alike in any order
        table, held, refs = ref.fork(table, held, refs, p, None, 16)
    assert s.h.tolist() == held.tolist() and s.r.tolist() == refs.tolist()
    for b, m in enumerate(held):
        assert s.t[b, :m].tolist() == table[b, :m].tolist()
