"""Private pages, forked sequences and compaction of a pool against plain host implementations."""
import numpy as np
import pytest
import torch

import cache8_ref as ref
from paper_2608_12703_gb300 import asrspec as A

pytestmark = pytest.mark.gpu

DT = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16, "fp8": torch.float8_e4m3fn}


def i32(x):
    return torch.tensor(np.asarray(x, dtype=np.int32), device="cuda")


def raw(x):
    return x.contiguous().view(torch.uint8)


class State:
    """A pool in use: `groups` of sequences that share the pages of their common part, pages scattered over the pool."""

    def __init__(self, seed, groups, page, width, spare, dtype="bf16", layers=2, kv_heads=2, dim=64, layout="head"):
        from paper_2608_12703_gb300 import serving
        rng = np.random.default_rng(seed)
        lens = [n for lens, _ in groups for n in lens]
        held = [-(-n // page) for n in lens]
        live = sum(sum(-(-n // page) for n in lens) - (len(lens) - 1) * common for lens, common in groups)
        n_pages = live + spare
        order = rng.permutation(n_pages)
        table = rng.integers(0, n_pages, (len(lens), width)).astype(np.int32)    # what is not held may be anything
        refs, at, b = np.zeros(n_pages, np.int32), 0, 0
        for group, common in groups:
            first = b
            for n in group:
                h = -(-n // page)
                s = common if b > first else 0
                table[b, :s] = table[first, :s]
                table[b, s:h] = order[at:at + h - s]
                at += h - s
                np.add.at(refs, table[b, :h], 1)
                b += 1
        assert at == live
        self.page, self.lens, self.live = page, lens, live
        self.table, self.held, self.refs = table, np.array(held, np.int32), refs
        self.t, self.h, self.r = i32(table), i32(held), i32(refs)
        g = torch.Generator(device="cuda").manual_seed(seed)
        shape = (n_pages, kv_heads, page, dim) if layout == "head" else (n_pages, page, kv_heads, dim)
        caches, self.arrays = [], []
        for _ in range(layers):
            pages = [torch.randn(shape, generator=g, device="cuda").to(DT[dtype]) for _ in range(2)]
            if layout != "head":
                pages = [x.transpose(1, 2) for x in pages]
            self.arrays += [(x, 1) for x in pages]
            if dtype == "fp8":
                scales = [torch.rand((n_pages, kv_heads, page // 16), generator=g, device="cuda") for _ in range(2)]
                self.arrays += [(x, 16) for x in scales]
                caches.append(serving.PagedCache8(*pages, *scales, self.t))
            else:
                caches.append(serving.PagedCache(*pages, self.t))
        self.before = [x.clone() for x, _ in self.arrays]
        self.pool = serving.PagePool(caches, self.h, self.r)

    def outs(self, in_place):
        """Outputs of the calls, filled with a mark."""
        if in_place:
            return {}
        return dict(table_out=torch.full_like(self.t, -7), held_out=torch.full_like(self.h, -7), refs_out=torch.full_like(self.r, -7))

    def check_copies(self, copies):
        for (x, slots), old in zip(self.arrays, self.before):
            want = old.clone()
            for src, dst, n in copies:
                n = self.page if n is None else n
                rows = -(-n // slots)
                want[dst][:, :rows] = old[src][:, :rows]
            assert torch.equal(raw(x), raw(want))

    def check_table(self, got, want, held, in_place):
        got = got.cpu().numpy()
        for b, n in enumerate(held):
            assert (got[b, :n] == want[b, :n]).all(), b
            assert (got[b, n:] == (self.table[b, n:] if in_place else -7)).all()    # the rest is left as it is

    def reserve(self, rows, in_place, lens=None):
        lens = self.lens if lens is None else lens
        outs = self.outs(in_place)
        table, held, refs, counts = self.pool.reserve(i32(lens), i32(rows), **outs)
        assert self.pool.status() == 0
        wt, wh, wr, wc, copies = ref.reserve(self.table, self.held, self.refs, lens, rows, self.page)
        assert held.tolist() == wh.tolist() and refs.tolist() == wr.tolist() and counts.tolist() == list(wc)
        self.check_table(table, wt, wh, in_place)
        self.check_copies(copies)
        return copies


def samples(n, length, page):
    """n samples of a prompt right after the fork: all pages shared."""
    return ([length] * n, -(-length // page))


@pytest.mark.parametrize("in_place", [True, False])
@pytest.mark.parametrize("dtype,page,layout", [("bf16", 16, "head"), ("fp32", 48, "slot"), ("fp8", 32, "head"), ("fp8", 64, "slot"),
                                               ("fp16", 128, "head")])
def test_reserve_matches_plain(built_lib, cuda, dtype, page, layout, in_place):
    groups = [samples(4, 3 * page + 5, page), samples(1, page, page), samples(3, 2 * page, page), samples(2, 1, page),
              ([2 * page + 1, 2 * page + 9, 2 * page + 1], 2), ([page - 1], 0), ([0], 0), samples(5, 17, page)]
    n = sum(len(g) for g, _ in groups)
    s = State(1 + page, groups, page, 8, 60, dtype, layout=layout)
    copies = s.reserve([(i * 7) % 20 for i in range(n)], in_place)
    assert copies


@pytest.mark.parametrize("in_place", [True, False])
def test_reserve_behind_a_rollback(built_lib, cuda, in_place):
    """Sequences that hold more pages than their length needs, shared ones among them: every touched page becomes private."""
    page = 16
    s = State(3, [samples(3, 100, page), ([90, 100], 6), samples(2, 64, page)], page, 10, 30)
    s.reserve([40, 1, 0, 16, 33, 5, 60], in_place, lens=[20, 97, 50, 90, 37, 0, 64])


@pytest.mark.parametrize("in_place", [True, False])
def test_reserve_prompts_and_most_sequences(built_lib, cuda, in_place):
    """Many pages at once; 1024 sequences; a pool of more pages than a block counts."""
    s = State(4, [samples(2, 5, 16), ([0], 0), ([33], 0)], 16, 700, 2100, layers=1)
    s.reserve([10000, 0, 11000, 7000], in_place)
    s = State(5, [samples(8, (i * 11) % 60, 16) for i in range(128)], 16, 6, 9000, layers=1, kv_heads=1)
    s.reserve([(i * 5) % 30 for i in range(1024)], in_place)
    s = State(6, [samples(2, 40, 16)], 16, 5000, 40000, layers=1, kv_heads=1)
    s.reserve([30, 70000], in_place)


@pytest.mark.parametrize("in_place", [True, False])
def test_reserve_without_room(built_lib, cuda, in_place):
    """A page too few: nothing changes, the status says so, and so do the counts."""
    s = State(7, [samples(3, 20, 16), samples(1, 16, 16)], 16, 6, 3)
    outs = s.outs(in_place)
    table, held, refs, counts = s.pool.reserve(i32(s.lens), i32([5, 5, 20, 1]), **outs)
    assert s.pool.status() == A.ST_CAPACITY
    s.check_table(table, s.table, s.held, in_place)
    assert held.tolist() == s.held.tolist() and refs.tolist() == s.refs.tolist() and counts.tolist() == [0, 3]
    s.check_copies([])
    s.reserve([5, 5, 4, 0], in_place)


def test_reserve_twice_and_data_errors(built_lib, cuda):
    s = State(8, [samples(2, 20, 16), samples(2, 30, 16), ([40], 0)], 16, 4, 10)
    s.reserve([1] * 5, True)
    table, held, refs = s.t.clone(), s.h.clone(), s.r.clone()
    _, _, _, counts = s.pool.reserve(i32(s.lens), i32([1] * 5))      # all private by now
    assert counts[0] == 0 and torch.equal(table, s.t) and torch.equal(held, s.h) and torch.equal(refs, s.r)
    # lengths past what is held, rows below zero, more than the table has room for
    _, _, _, counts = s.pool.reserve(i32([33, -1, 30, 30, 40]), i32([1, 1, -1, 100, 0]))
    assert s.pool.status() == A.ST_BAD_LENS | A.ST_CAPACITY and counts[0] == 0
    assert torch.equal(table, s.t) and torch.equal(held, s.h) and torch.equal(refs, s.r)
    s.t[4, 2] = 10 ** 6      # a bad page counts as the sequence's own
    _, _, _, counts = s.pool.reserve(i32([20, 20, 30, 30, 40]), i32([0, 0, 0, 0, 20]))
    assert s.pool.status() == A.ST_BOUNDS and counts[0] == 1 and int(s.t[4, 2]) == 10 ** 6 and int(s.h[4]) == 4


@pytest.mark.parametrize("in_place", [True, False])
@pytest.mark.parametrize("seed", range(3))
def test_fork_matches_plain(built_lib, cuda, seed, in_place):
    rng = np.random.default_rng(seed)
    groups = [samples(4, 100, 16), samples(1, 16, 16), ([200, 170, 165], 10), ([0, 0], 0), samples(2, 1, 16)]
    for parent, keep in ((True, False), (True, True), (False, True)):
        s = State(seed, groups, 16, 20, 5)
        n = len(s.lens)
        s.refs[3] += 2      # a holder of the caller's own
        s.r[3] += 2
        p = [int(x) for x in rng.integers(-1, n, n)] if parent else None
        k = [int(x) for x in rng.integers(0, 250, n)] if keep else None
        outs = s.outs(in_place)
        table, held, refs = s.pool.fork(None if p is None else i32(p), None if k is None else i32(k), **outs)
        assert s.pool.status() == 0
        wt, wh, wr = ref.fork(s.table, s.held, s.refs, p, k, 16)
        assert held.tolist() == wh.tolist() and refs.tolist() == wr.tolist()
        s.check_table(table, wt, wh, in_place)
        s.check_copies([])


@pytest.mark.parametrize("in_place", [True, False])
def test_fork_long_rows(built_lib, cuda, in_place):
    s = State(9, [([50000, 40000, 49000], 1000), ([30000], 0)], 16, 5000, 7, layers=1, kv_heads=1)
    table, held, refs = s.pool.fork(i32([1, 0, 3, -1]), i32([45000, 49990, 50, 0]), **s.outs(in_place))
    wt, wh, wr = ref.fork(s.table, s.held, s.refs, [1, 0, 3, -1], [45000, 49990, 50, 0], 16)
    assert held.tolist() == wh.tolist() and refs.tolist() == wr.tolist()
    s.check_table(table, wt, wh, in_place)


@pytest.mark.parametrize("in_place", [True, False])
def test_fork_data_errors(built_lib, cuda, in_place):
    s = State(10, [samples(2, 40, 16), ([20, 50], 1)], 16, 5, 4)
    table, held, refs = s.pool.fork(i32([9, -2, 3, 0]), i32([5, 5, -1, 17]), **s.outs(in_place))
    assert s.pool.status() == A.ST_BOUNDS | A.ST_BAD_LENS
    wt, wh, wr = ref.fork(s.table, s.held, s.refs, [0, 1, 2, 0], [99, 99, 99, 17], 16)
    assert held.tolist() == wh.tolist() and refs.tolist() == wr.tolist()
    s.check_table(table, wt, wh, in_place)


@pytest.mark.parametrize("in_place", [True, False])
@pytest.mark.parametrize("dtype,page,layout,spare", [("bf16", 16, "head", 9), ("fp32", 48, "slot", 0), ("fp8", 32, "head", 40),
                                                     ("fp8", 64, "slot", 3), ("fp16", 16, "head", 9000), ("fp8", 16, "head", 20000)])
def test_compact_matches_plain(built_lib, cuda, dtype, page, layout, spare, in_place):
    groups = [samples(3, 100, page), ([200, 170], 2), ([0], 0), samples(2, 16, page)]
    if spare > 1000:
        groups += [([20000], 0), ([50000], 0)]
    s = State(spare, groups, page, 4000, spare, dtype, layers=1 if spare > 1000 else 2, layout=layout)
    outs = s.outs(in_place)
    outs.pop("held_out", None)
    table, refs, where, live = s.pool.compact(**outs)
    assert s.pool.status() == 0
    wt, wr, ww, wl, moves = ref.compact(s.table, s.held, s.refs)
    assert refs.tolist() == wr.tolist() and where.tolist() == ww.tolist() and live.tolist() == [wl]
    s.check_table(table, wt, s.held, in_place)
    s.check_copies([(a, b, None) for a, b in moves])


@pytest.mark.parametrize("n", [8191, 8192, 8193, 16384])
def test_compact_edges_of_chunks(built_lib, cuda, n):
    """All pages live, none, one at the end, and as many as a block looks at."""
    from paper_2608_12703_gb300 import serving
    k = torch.zeros((n, 1, 16, 64), dtype=torch.float8_e4m3fn, device="cuda")
    sc = torch.arange(n, dtype=torch.float32, device="cuda").reshape(n, 1, 1)
    t = torch.full((1, n), n - 1, dtype=torch.int32, device="cuda")
    for refs in (np.ones(n), np.zeros(n), np.arange(n) == n - 1, np.arange(n) % 2, np.arange(n) < n // 2):
        refs = refs.astype(np.int32)
        s = sc.clone()
        held = int(refs[-1])
        pool = serving.PagePool(serving.PagedCache8(k, k.clone(), s, s.clone(), t.clone()), i32([held]), i32(refs))
        table, now, where, live = pool.compact()
        wt, wr, ww, wl, moves = ref.compact(t.cpu().numpy(), np.array([held]), refs)
        assert now.tolist() == wr.tolist() and where.tolist() == ww.tolist() and int(live) == wl
        assert int(table[0, 0]) == wt[0, 0]
        want = sc.clone()
        for a, b in moves:
            want[b] = sc[a]
        assert torch.equal(s, want) and pool.status() == 0


def test_side_stream_and_graph(built_lib, cuda):
    """A captured reserve and compact replayed beside eager calls on another stream; workspaces are apart."""
    s = State(11, [samples(3, 40, 16), samples(2, 20, 16)], 16, 6, 12)
    lens, rows = i32(s.lens), i32([3] * 5)
    want = [x.clone() for x in s.pool.reserve(lens, rows, **s.outs(False))]
    graph, outs = torch.cuda.CUDAGraph(), s.outs(False)
    with torch.cuda.graph(graph):
        got = s.pool.reserve(lens, rows, **outs)
        moved = s.pool.compact(table_out=torch.empty_like(s.t), refs_out=torch.empty_like(s.r))
    side = torch.cuda.Stream()
    for _ in range(3):
        for x in outs.values():
            x.fill_(-7)
        side.wait_stream(torch.cuda.current_stream())
        graph.replay()
        with torch.cuda.stream(side):
            other = s.pool.fork(i32([1, 0, 2, 4, 3]), **s.outs(False))
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            assert torch.equal(a, b)
        assert int(moved[3]) == s.live
        wt, wh, wr = ref.fork(s.table, s.held, s.refs, [1, 0, 2, 4, 3], None, 16)
        assert other[2].tolist() == wr.tolist()
        # the compaction has moved pages while the table stayed: put them back
        for (x, _), old in zip(s.arrays, s.before):
            x.copy_(old)
    assert s.pool.status() == 0


def test_refusals(built_lib, cuda):
    from paper_2608_12703_gb300 import serving
    s = State(12, [samples(2, 20, 16)], 16, 4, 4)
    lens, rows = i32(s.lens), i32([1, 1])
    for a, kw in (((None, rows), {}), ((lens, None), {}), ((lens.long(), rows), {}), ((lens[:1], rows), {}), ((lens.cpu(), rows), {}),
                  ((lens, rows), dict(table_out=s.t[:, :3])), ((lens, rows), dict(table_out=torch.empty((4, 2), dtype=torch.int32, device="cuda").T)),
                  ((lens, rows), dict(held_out=s.r)), ((lens, rows), dict(refs_out=s.r.float()))):
        with pytest.raises(A.AsrSpecError, match="required|contiguous"):
            s.pool.reserve(*a, **kw)
    with pytest.raises(A.AsrSpecError):
        s.pool.fork(lens.float())
    with pytest.raises(A.AsrSpecError):
        s.pool.fork(lens, 5)
    with pytest.raises(A.AsrSpecError):
        s.pool.compact(refs_out=s.h)
    c = s.pool.caches[0]
    other = serving.PagedCache(c.k_pages, c.v_pages, s.t.clone())
    for caches, held, refs in (([], s.h, s.r), ([c, other], s.h, s.r), ([c, 3], s.h, s.r), ([c], s.r, s.r), ([c], s.h, s.r[:-1]),
                               ([c], s.h.long(), s.r)):
        with pytest.raises(A.AsrSpecError):
            serving.PagePool(caches, held, refs)
    assert s.pool.status() == 0


def test_offsets_past_32_bits(built_lib, cuda):
    """A pool of more than 4 GB: copies from its last pages to others of them, and to its front."""
    from paper_2608_12703_gb300 import serving
    page, n_pages = 16, (9 << 29) // (16 * 64 * 2)
    k, v = (torch.empty((n_pages, 1, page, 64), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    refs = torch.full((n_pages,), 1, dtype=torch.int32, device="cuda")      # all others are in use
    a, b, c = n_pages - 1, n_pages - 2, n_pages - 3
    refs[a], refs[b], refs[c], refs[5] = 2, 0, 2, 0
    table = i32([[c, a, 0], [c, a, 0]])
    held = i32([2, 2])
    k[a], v[a] = 3.0, 4.0
    k[c], v[c] = 5.0, 6.0
    pool = serving.PagePool(serving.PagedCache(k, v, table), held, refs)
    counts = pool.reserve(i32([20, 20]), i32([1, 1]))[3]
    # two share the last page and both write: the lower one keeps it, the other takes the lowest free page
    assert counts.tolist() == [1, 1] and table[:, 1].tolist() == [a, 5] and int(refs[a]) == 1 and int(refs[5]) == 1
    assert bool((k[5, :, :4] == 3.0).all()) and bool((v[5, :, :4] == 4.0).all())
    where, live = pool.compact()[2:]
    assert int(live) == n_pages - 1 and int(where[a]) == b and table.tolist()[0][:2] == [c, b] and table.tolist()[1][:2] == [c, 5]
    assert bool((k[b, :, :4] == 3.0).all()) and bool((k[c] == 5.0).all()) and refs[-4:].tolist() == [1, 2, 1, 0]
    assert pool.status() == 0
