"""The functions of the binding with the library's names, for an 8-bit cache, pools and logits, give what the classes over them
give; pools of many caches."""
import ctypes

import numpy as np
import pytest
import torch

import cache8_ref as ref
from paper_2608_12703_gb300 import asrspec as A
from test_gpu_cache8 import codes, fill, gen, i32, make_rows, pool, same_bits
from test_gpu_pool import State, raw, samples

pytestmark = pytest.mark.gpu


def stream():
    return torch.cuda.current_stream().cuda_stream


def zeros(n):
    return torch.zeros(n, dtype=torch.uint8, device="cuda")


def test_cache(built_lib, cuda):
    from paper_2608_12703_gb300 import serving
    g, lens, R = gen(90), [60, 33, 0], 4
    k, v, ks, vs, table = pool(g, 2, 64, 16, [n + R for n in lens])
    fill(g, k, ks, table, lens)
    fill(g, v, vs, table, lens)
    q, kn, vn = make_rows(g, 3, R, 4, 2, 64, torch.bfloat16, True)
    n, m = i32(lens), i32([4, 2, 3])
    other = [x.clone() for x in (k, v, ks, vs)]
    want = serving.PagedCache8(*other, table).attend(q, n, k_new=kn, v_new=vn, rows=m)
    c = A.AsrPaged8Cache(k.data_ptr(), v.data_ptr(), *k.stride()[:3], ks.data_ptr(), vs.data_ptr(), *ks.stride()[:2], table.data_ptr(),
                         table.stride(0), k.shape[0], 16, table.shape[1], 2, 64, 3, None)
    rows = A.AsrPagedRows(q.data_ptr(), *q.stride()[:3], kn.data_ptr(), vn.data_ptr(), *kn.stride()[:3], n.data_ptr(), m.data_ptr(),
                          R, 4, 1, 0.125)
    A.asr_spec_paged8_append(ctypes.byref(c), rows, 1, stream())
    assert torch.equal(codes(k), codes(other[0])) and torch.equal(codes(v), codes(other[1]))
    assert same_bits(ks, other[2]) and same_bits(vs, other[3])
    ws = zeros(built_lib.asr_spec_paged8_attend_ws(ctypes.byref(c), ctypes.byref(rows), 1))
    out, lse = torch.zeros_like(want[0]), torch.zeros_like(want[1])
    A.asr_spec_paged8_attend(ctypes.byref(c), rows, 1, out, lse, ws, ws.numel(), stream())
    assert same_bits(out, want[0]) and same_bits(lse, want[1])
    with pytest.raises(A.AsrSpecError, match="CAPACITY"):
        A.asr_spec_paged8_attend(ctypes.byref(c), rows, 1, out, lse, ws, ws.numel() - 1, stream())


def arrays_of(s):
    return [A.AsrPageArray(x.data_ptr(), *(t * x.element_size() for t in x.stride()[:3]), x.shape[1], x.shape[2],
                           x.element_size() * (x.shape[3] if x.dim() == 4 else 1), slots) for x, slots in s.arrays]


def test_pool(built_lib, cuda):
    s = State(91, [samples(3, 40, 16), samples(2, 21, 16), ([60], 0)], 16, 8, 20, "fp8")
    B = len(s.lens)
    i = [torch.full_like(x, -7) for x in (s.t, s.h, s.r)]
    p = A.AsrPagePool(s.t.data_ptr(), 8, s.h.data_ptr(), s.r.data_ptr(), i[0].data_ptr(), 8, i[1].data_ptr(), i[2].data_ptr(), s.r.numel(),
                      16, 8, B, None)
    plan = torch.from_numpy(A.asr_spec_pool_plan(arrays_of(s), 16)).cuda()
    ws, n = zeros(built_lib.asr_spec_pool_ws(ctypes.byref(p))), len(s.arrays)
    parent, keep = [1, 0, 0, 4, 4, 2], [30, 100, 0, 20, 5, 39]
    A.asr_spec_pool_fork(p, i32(parent), i32(keep), ws, ws.numel(), stream())
    wt, wh, wr = ref.fork(s.table, s.held, s.refs, parent, keep, 16)
    assert i[1].tolist() == wh.tolist() and i[2].tolist() == wr.tolist()
    s.check_table(i[0], wt, wh, False)
    counts, rows = torch.zeros(2, dtype=torch.int32, device="cuda"), [3, 0, 9, 20, 1, 5]
    A.asr_spec_pool_reserve(p, plan, n, i32(s.lens), i32(rows), counts, ws, ws.numel(), stream())
    wt, wh, wr, wc, copies = ref.reserve(s.table, s.held, s.refs, s.lens, rows, 16)
    assert i[1].tolist() == wh.tolist() and i[2].tolist() == wr.tolist() and counts.tolist() == list(wc)
    s.check_copies(copies)
    for (x, _), old in zip(s.arrays, s.before):
        x.copy_(old)
    where, live = torch.zeros_like(s.r), torch.zeros(1, dtype=torch.int32, device="cuda")
    A.asr_spec_pool_compact(p, plan, n, where, live, ws, ws.numel(), stream())
    wt, wr, ww, wl, moves = ref.compact(s.table, s.held, s.refs)
    assert i[2].tolist() == wr.tolist() and where.tolist() == ww.tolist() and live.tolist() == [wl]
    s.check_copies([(a, b, None) for a, b in moves])
    with pytest.raises(A.AsrSpecError, match="CAPACITY"):
        A.asr_spec_pool_fork(p, None, None, ws, ws.numel() - 1, stream())


def test_logits(built_lib, cuda):
    from paper_2608_12703_gb300 import serving
    g = gen(92)
    x = torch.randn((2, 3, 70), generator=g, device="cuda")
    history, draft = (torch.randint(0, 70, n, generator=g, device="cuda").int() for n in ((2, 9), (2, 2)))
    want = serving.adjust_logits(x, history=history, draft=draft, repetition=1.5, frequency=0.25, presence=-0.5, out=torch.zeros_like(x))
    out = torch.zeros_like(x)
    r = A.AsrLogitRules(logits=x.data_ptr(), batch_stride=210, row_stride=70, out=out.data_ptr(), out_batch_stride=210, out_row_stride=70,
                        batch=2, rows=3, vocab=70, dtype=0, history=history.data_ptr(), history_stride=9, history_max=9,
                        draft=draft.data_ptr(), repetition_all=1.5, frequency_all=0.25, presence_all=-0.5)
    A.asr_spec_adjust_logits(r, stream())
    assert torch.equal(out, want)
    r.rows = 33
    with pytest.raises(A.AsrSpecError, match="INVAL"):
        A.asr_spec_adjust_logits(r, stream())


class Layers(State):
    """As a State, with caches of several types and numbers of heads: arrays of different numbers of tasks."""

    def __init__(self, seed, groups, page, width, spare, layers):
        from paper_2608_12703_gb300 import serving
        super().__init__(seed, groups, page, width, spare, layers=1, kv_heads=1)
        g, n, caches, self.arrays = torch.Generator(device="cuda").manual_seed(seed), self.r.numel(), [], []
        for i in range(layers):
            heads, dim = (1, 7, 2, 13, 3)[i % 5], (64, 128)[i % 3 == 2]
            dtype = (torch.float8_e4m3fn, torch.bfloat16, torch.float8_e4m3fn, torch.float32)[i % 4]
            pages = [torch.randn((n, heads, page, dim), generator=g, device="cuda").to(dtype) for _ in range(2)]
            self.arrays += [(x, 1) for x in pages]
            if dtype == torch.float8_e4m3fn:
                scales = [torch.rand((n, heads, page // 16), generator=g, device="cuda") for _ in range(2)]
                self.arrays += [(x, 16) for x in scales]
                caches.append(serving.PagedCache8(*pages, *scales, self.t))
            else:
                caches.append(serving.PagedCache(*pages, self.t))
        self.before = [x.clone() for x, _ in self.arrays]
        self.pool = serving.PagePool(caches, self.h, self.r)


@pytest.mark.parametrize("layers,page", [(11, 16), (12, 32), (21, 16), (33, 32), (340, 16), (341, 16)])
def test_pools_of_many_caches(built_lib, cuda, layers, page):
    """34 to 1024 arrays, as many as there may be: each array's part of a page goes along."""
    s = Layers(93 + layers, [samples(3, 2 * page + 5, page), samples(2, 9, page), ([page, 3 * page - 1], 1)], page, 6, 12, layers)
    assert len(s.arrays) == 2 * layers + 2 * -(-layers // 2)
    assert s.reserve([1, 20, 3, 2, 5, 4, 2], False)
    for (x, _), old in zip(s.arrays, s.before):
        x.copy_(old)
    where, live = s.pool.compact(table_out=torch.empty_like(s.t), refs_out=torch.empty_like(s.r))[2:]
    ww, wl, moves = ref.compact(s.table, s.held, s.refs)[2:]
    assert where.tolist() == ww.tolist() and live.tolist() == [wl] and moves and s.pool.status() == 0
    s.check_copies([(a, b, None) for a, b in moves])


def test_too_many_arrays(built_lib, cuda):
    from paper_2608_12703_gb300 import serving
    s = State(94, [samples(2, 20, 16)], 16, 4, 4, "fp8", layers=1)
    c = s.pool.caches[0]
    with pytest.raises(A.AsrSpecError, match="1024"):
        serving.PagePool([c] * 257, s.h, s.r)
    assert np.array_equal(raw(s.arrays[0][0]).cpu().numpy(), raw(s.before[0]).cpu().numpy())


def test_an_expanded_history_is_refused(built_lib, cuda):
    """Rows of a history lie apart; one for all utterances is made contiguous first."""
    from paper_2608_12703_gb300 import serving
    x = torch.randn((3, 2, 50), generator=gen(95), device="cuda")
    h = torch.arange(7, dtype=torch.int32, device="cuda")
    with pytest.raises(A.AsrSpecError, match="contiguous"):
        serving.adjust_logits(x, history=h.expand(3, 7), repetition=2.0, out=torch.zeros_like(x))
    got = serving.adjust_logits(x, history=h.expand(3, 7).contiguous(), repetition=2.0, out=torch.zeros_like(x))
    want = x.clone()
    want[:, :, :7] = torch.where(want[:, :, :7] > 0, want[:, :, :7] / 2, want[:, :, :7] * 2)
    assert torch.equal(got, want)
