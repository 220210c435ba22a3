"""Argument checks of the handle-free entry points, at the C ABI, without a GPU:
every call here is refused before anything is launched."""
import ctypes

import pytest

from paper_2608_12703_gb300 import asrspec as A

INVAL, CAPACITY = -1, -3


def cache(**kw):
    f = dict(k_pages=4096, v_pages=8192, page_stride=2 * 16 * 64, head_stride=16 * 64, slot_stride=64, page_table=256,
             table_stride=8, n_pages=10, page_size=16, max_pages=8, kv_heads=2, head_dim=64, batch=3, dtype=1, status=None)
    f.update(kw)
    return A.AsrPagedCache(**f)


def rows(**kw):
    f = dict(q=4096, q_batch_stride=512, q_row_stride=256, q_head_stride=64, k_new=None, v_new=None, new_batch_stride=0,
             new_row_stride=0, new_head_stride=0, kv_len=64, rows=None, max_rows=2, heads=4, causal=1, scale=0.125)
    f.update(kw)
    return A.AsrPagedRows(**f)


def scores(**kw):
    f = dict(score=256, pos=None, batch_stride=256, head_stride=128, slots=128, score_out=256, pos_out=None,
             out_batch_stride=256, out_head_stride=128, slots_out=128, first_pos=None)
    f.update(kw)
    return A.AsrPagedScores(**f)


def logits(**kw):
    f = dict(target=4096, target_batch_stride=400, target_row_stride=100, draft_logits=None, draft_batch_stride=0,
             draft_row_stride=0, batch=2, k=3, vocab=100, dtype=0)
    f.update(kw)
    return A.AsrSampledLogits(**f)


BAD_CACHE = [dict(k_pages=None), dict(v_pages=None), dict(page_table=None), dict(dtype=3), dict(head_dim=80), dict(batch=0),
             dict(batch=1025), dict(kv_heads=0), dict(n_pages=0), dict(page_size=0), dict(page_size=24), dict(max_pages=0),
             dict(max_pages=1 << 28), dict(table_stride=7), dict(k_pages=4104), dict(page_stride=2047), dict(head_stride=-16),
             dict(slot_stride=32), dict(slot_stride=68), dict(status=2)]
BAD_ROWS = [dict(q=None), dict(kv_len=None), dict(k_new=4096), dict(k_new=4096, v_new=4096, causal=0), dict(max_rows=0),
            dict(max_rows=5000), dict(heads=3), dict(heads=0), dict(scale=0.0), dict(scale=float("nan")),
            dict(scale=float("inf")), dict(q=4100), dict(q_row_stride=255), dict(q_batch_stride=-512), dict(rows=2),
            dict(k_new=4096, v_new=4096, new_row_stride=4)]


@pytest.fixture(scope="module")
def L(built_lib):
    return built_lib


def ref(x):
    return ctypes.byref(x)


@pytest.mark.parametrize("bad", BAD_CACHE + [None], ids=str)
def test_cache_refusals(L, bad):
    c = None if bad is None else ref(cache(**bad))
    assert L.asr_spec_paged_attend(c, ref(rows()), 4096, None, 4096, 1 << 30, None) == INVAL
    assert L.asr_spec_paged_attend_ws(c, ref(rows())) == INVAL
    assert L.asr_spec_paged_weigh(c, ref(rows()), ref(scores()), 256, 8, 4, None) == INVAL
    assert L.asr_spec_paged_evict(c, ref(scores(pos=256, pos_out=256)), 64, 64, 8, 0, 0, 64, 256, 1 << 30, None) == INVAL
    assert L.asr_spec_paged_evict_ws(c, ref(scores()), 8) == INVAL


@pytest.mark.parametrize("bad", BAD_ROWS + [None], ids=str)
def test_rows_refusals(L, bad):
    r = None if bad is None else ref(rows(**bad))
    assert L.asr_spec_paged_attend(ref(cache()), r, 4096, None, 4096, 1 << 30, None) == INVAL
    assert L.asr_spec_paged_attend_ws(ref(cache()), r) == INVAL
    assert L.asr_spec_paged_weigh(ref(cache()), r, ref(scores()), 256, 8, 4, None) == INVAL


def test_attend_outputs_and_workspace(L):
    c, r = cache(), rows()
    assert L.asr_spec_paged_attend(ref(c), ref(r), None, None, 4096, 1 << 30, None) == INVAL
    assert L.asr_spec_paged_attend(ref(c), ref(r), 4100, None, 4096, 1 << 30, None) == INVAL
    assert L.asr_spec_paged_attend(ref(c), ref(r), 4096, 2, 4096, 1 << 30, None) == INVAL
    assert L.asr_spec_paged_attend(ref(c), ref(r), 4096, None, None, 1 << 30, None) == INVAL
    n = L.asr_spec_paged_attend_ws(ref(c), ref(r))
    assert n > 0
    assert L.asr_spec_paged_attend(ref(c), ref(r), 4096, None, 4096, n - 1, None) == CAPACITY


@pytest.mark.parametrize("bad", [dict(score_out=None), dict(slots=0), dict(head_stride=127), dict(pos=256), dict(score=2),
                                 dict(first_pos=4)], ids=str)
def test_weigh_refusals(L, bad):
    assert L.asr_spec_paged_weigh(ref(cache()), ref(rows()), ref(scores(**bad)), 256, 8, 4, None) == INVAL
    assert L.asr_spec_paged_weigh(ref(cache()), ref(rows()), ref(scores()), None, 8, 4, None) == INVAL


@pytest.mark.parametrize("bad", [dict(score=None), dict(score_out=None), dict(pos=None), dict(pos_out=None), dict(slots=0),
                                 dict(slots_out=0), dict(out_head_stride=100), dict(head_stride=100), dict(pos=257)], ids=str)
def test_evict_refusals(L, bad):
    s = scores(**{**dict(pos=256, pos_out=256), **bad})
    assert L.asr_spec_paged_evict(ref(cache()), ref(s), 64, 64, 8, 0, 0, 64, 256, 1 << 30, None) == INVAL


def test_evict_numbers_and_workspace(L):
    c, s = cache(), scores(pos=256, pos_out=256)
    for budget, recent, first in ((0, 0, 0), (8, -1, 0), (8, 0, -1)):
        assert L.asr_spec_paged_evict(ref(c), ref(s), 64, 64, budget, recent, first, 64, 256, 1 << 30, None) == INVAL
    for a in ((None, 64, 64), (64, None, 64), (64, 64, None)):
        assert L.asr_spec_paged_evict(ref(c), ref(s), a[0], a[1], 8, 0, 0, a[2], 256, 1 << 30, None) == INVAL
    n = L.asr_spec_paged_evict_ws(ref(c), ref(s), 8)
    assert n > 0
    assert L.asr_spec_paged_evict(ref(c), ref(s), 64, 64, 8, 0, 0, 64, 256, n - 1, None) == CAPACITY


@pytest.mark.parametrize("bad", [dict(target=None), dict(dtype=3), dict(batch=0), dict(k=-1), dict(k=32), dict(vocab=0),
                                 dict(target_row_stride=99), dict(target=4098), dict(draft_logits=4096),
                                 dict(draft_logits=4097, draft_row_stride=100)], ids=str)
def test_accept_refusals(L, bad):
    args = [64, 64, 64, 64, 100, 1.0, 64, 64, 64, 64, None, None]
    assert L.asr_spec_accept_sampled(ref(logits(**bad)), *args) == INVAL


@pytest.mark.parametrize("at,value", [(0, None), (2, None), (3, None), (4, 99), (5, 0.0), (5, -1.0), (5, float("nan")),
                                      (5, float("inf")), (6, None), (7, None), (8, None), (9, None), (3, 66), (10, 2)])
def test_accept_argument_refusals(L, at, value):
    args = [64, 64, 64, 64, 100, 1.0, 64, 64, 64, 64, None, None]
    args[at] = value
    assert L.asr_spec_accept_sampled(ref(logits()), *args) == INVAL


def test_tensors_must_be_on_a_gpu():
    import torch
    from paper_2608_12703_gb300 import serving
    with pytest.raises(A.AsrSpecError, match="ASR_E_INVAL"):
        serving.PagedCache(torch.zeros(2, 2, 16, 64), torch.zeros(2, 2, 16, 64), torch.zeros(1, 2, dtype=torch.int32))
    with pytest.raises(A.AsrSpecError, match="ASR_E_INVAL"):
        serving.accept_sampled(torch.zeros(1, 2, 8), torch.zeros(1, 1, dtype=torch.int32), None, torch.zeros(1, 1), torch.ones(1, 8))
