"""Argument checks of the entry points over an 8-bit paged cache, of pools and of logits, at the C ABI, without a GPU:
every call here is refused before anything is launched."""
import ctypes

import numpy as np
import pytest

from paper_2608_12703_gb300 import asrspec as A

INVAL, CAPACITY = -1, -3
BIG = 1 << 40


def ref(x):
    return None if x is None else ctypes.byref(x)


def made(kind, base, kw):
    return kind(**{**base, **kw})


def cache(**kw):
    return made(A.AsrPaged8Cache, dict(
        k_pages=4096, v_pages=8192, page_stride=2 * 32 * 64, head_stride=32 * 64, slot_stride=64, k_scale=256, v_scale=512,
        scale_page_stride=4, scale_head_stride=2, page_table=256, table_stride=8, n_pages=10, page_size=32, max_pages=8, kv_heads=2,
        head_dim=64, batch=3, status=None), kw)


def rows(**kw):
    return made(A.AsrPagedRows, dict(
        q=4096, q_batch_stride=512, q_row_stride=256, q_head_stride=64, k_new=4096, v_new=4096, new_batch_stride=512,
        new_row_stride=128, new_head_stride=64, kv_len=64, rows=None, max_rows=2, heads=4, causal=1, scale=0.125), kw)


def pool(**kw):
    return made(A.AsrPagePool, dict(
        page_table=256, table_stride=8, held=64, refs=128, table_out=512, table_out_stride=8, held_out=64, refs_out=128, n_pages=10,
        page_size=32, max_pages=8, batch=3, status=None), kw)


def rules(**kw):
    return made(A.AsrLogitRules, dict(
        logits=4096, batch_stride=400, row_stride=100, out=8192, out_batch_stride=400, out_row_stride=100, batch=2, rows=4, vocab=100,
        dtype=0, history=64, history_stride=20, history_max=20, history_len=64, prompt_len=64, draft=64, lens=64, repetition=64,
        frequency=64, presence=64, repetition_all=1.0, frequency_all=0.0, presence_all=0.0, bias=64, bias_stride=100, mask=64,
        mask_batch_stride=16, mask_row_stride=4, status=None), kw)


@pytest.fixture(scope="module")
def L(built_lib):
    return built_lib


@pytest.mark.parametrize("bad", [
    dict(k_pages=None), dict(v_pages=None), dict(k_scale=None), dict(v_scale=None), dict(page_table=None), dict(head_dim=80),
    dict(batch=0), dict(batch=1025), dict(kv_heads=0), dict(kv_heads=1025), dict(n_pages=0), dict(page_size=0), dict(page_size=24),
    dict(max_pages=0), dict(max_pages=1 << 27), dict(table_stride=7), dict(k_pages=4104), dict(v_pages=8200), dict(page_stride=2056),
    dict(page_stride=0), dict(head_stride=-16), dict(slot_stride=32), dict(slot_stride=72), dict(slot_stride=1 << 27),
    dict(scale_page_stride=-1), dict(scale_head_stride=-2), dict(k_scale=258), dict(status=2), dict(page_table=3), None], ids=str)
def test_cache_refusals(L, bad):
    c = None if bad is None else ref(cache(**bad))
    assert L.asr_spec_paged8_attend(c, ref(rows()), 1, 4096, None, 4096, 1 << 30, None) == INVAL
    assert L.asr_spec_paged8_attend_ws(c, ref(rows()), 1) == INVAL
    assert L.asr_spec_paged8_append(c, ref(rows()), 1, None) == INVAL


@pytest.mark.parametrize("bad", [
    dict(q=None), dict(kv_len=None), dict(k_new=None), dict(causal=0), dict(max_rows=0), dict(max_rows=5000), dict(heads=3),
    dict(heads=0), dict(scale=0.0), dict(scale=float("nan")), dict(scale=float("inf")), dict(q=4100), dict(q_row_stride=255),
    dict(q_batch_stride=-512), dict(rows=2), dict(new_row_stride=4), dict(v_new=4100), None], ids=str)
def test_rows_refusals(L, bad):
    r = None if bad is None else ref(rows(**bad))
    assert L.asr_spec_paged8_attend(ref(cache()), r, 1, 4096, None, 4096, 1 << 30, None) == INVAL
    assert L.asr_spec_paged8_attend_ws(ref(cache()), r, 2) == INVAL


@pytest.mark.parametrize("bad", [dict(k_new=None), dict(v_new=None), dict(kv_len=None), dict(max_rows=0), dict(new_row_stride=4),
                                 dict(new_head_stride=-64), dict(k_new=4100), dict(rows=6), None], ids=str)
def test_append_refusals(L, bad):
    assert L.asr_spec_paged8_append(ref(cache()), None if bad is None else ref(rows(**bad)), 1, None) == INVAL


def test_attend_types_outputs_and_workspace(L):
    c, r = cache(), rows()
    for dtype in (0, 3, -1):
        assert L.asr_spec_paged8_attend(ref(c), ref(r), dtype, 4096, None, 4096, 1 << 30, None) == INVAL
        assert L.asr_spec_paged8_attend_ws(ref(c), ref(r), dtype) == INVAL
    for dtype in (3, -1):
        assert L.asr_spec_paged8_append(ref(c), ref(r), dtype, None) == INVAL
    for out, lse, ws in ((None, None, 4096), (4100, None, 4096), (4096, 2, 4096), (4096, None, None), (4096, None, 4100)):
        assert L.asr_spec_paged8_attend(ref(c), ref(r), 1, out, lse, ws, 1 << 30, None) == INVAL
    n = L.asr_spec_paged8_attend_ws(ref(c), ref(r), 1)
    assert n > 0
    assert L.asr_spec_paged8_attend(ref(c), ref(r), 1, 4096, None, 4096, n - 1, None) == CAPACITY


def pool_calls(L, p, plan=4096, n=1, ws=4096, size=1 << 40, a=64, b=64, c=64):
    yield L.asr_spec_pool_reserve(p, plan, n, a, b, c, ws, size, None)
    yield L.asr_spec_pool_compact(p, plan, n, a, b, ws, size, None)
    if plan == 4096 and n == 1 and a == b == c == 64:
        yield L.asr_spec_pool_fork(p, a, b, ws, size, None)


@pytest.mark.parametrize("bad", [
    dict(page_table=None), dict(held=None), dict(refs=None), dict(table_out=None), dict(refs_out=None), dict(batch=0), dict(batch=1025),
    dict(n_pages=0), dict(page_size=8), dict(page_size=40), dict(max_pages=0), dict(max_pages=1 << 27), dict(table_stride=7),
    dict(table_out_stride=7), dict(table_out=256, table_out_stride=9), dict(held=66), dict(refs_out=130), dict(status=1), None], ids=str)
def test_pool_refusals(L, bad):
    p = None if bad is None else ref(pool(**bad))
    assert all(rc == INVAL for rc in pool_calls(L, p))
    assert L.asr_spec_pool_ws(p) == INVAL


def test_pool_arguments(L):
    p = ref(pool())
    assert L.asr_spec_pool_reserve(ref(pool(held_out=None)), 4096, 1, 64, 64, 64, 4096, BIG, None) == INVAL
    assert L.asr_spec_pool_fork(ref(pool(held_out=None)), 64, 64, 4096, BIG, None) == INVAL
    for kw in (dict(n=-1), dict(n=1025), dict(plan=None), dict(plan=4100), dict(ws=None), dict(ws=4104), dict(a=None), dict(b=None),
               dict(a=66), dict(b=66)):
        assert all(rc == INVAL for rc in pool_calls(L, p, **kw)), kw
    assert L.asr_spec_pool_reserve(p, 4096, 1, 64, 64, None, 4096, BIG, None) == INVAL
    assert L.asr_spec_pool_fork(p, 66, None, 4096, BIG, None) == INVAL
    for large in (dict(n_pages=(1 << 30) + 1), dict(batch=1024, max_pages=(1 << 20) + 1, table_stride=1 << 21, table_out_stride=1 << 21)):
        assert all(rc == CAPACITY for rc in pool_calls(L, ref(pool(**large)))) and L.asr_spec_pool_ws(ref(pool(**large))) == CAPACITY
    n = L.asr_spec_pool_ws(p)
    assert n > 0 and all(rc == CAPACITY for rc in pool_calls(L, p, size=n - 1))


def array(**kw):
    return made(A.AsrPageArray, dict(base=4096, page_stride=8192, head_stride=4096, row_stride=128, heads=2, rows=32, row_bytes=128,
                                     row_slots=1), kw)


@pytest.mark.parametrize("bad", [
    dict(base=None), dict(base=4098), dict(page_stride=0), dict(page_stride=-16), dict(head_stride=0), dict(row_stride=124),
    dict(row_stride=130), dict(heads=0), dict(rows=0), dict(rows=16), dict(row_bytes=0), dict(row_bytes=126), dict(row_slots=0),
    dict(page_stride=1 << 41)], ids=str)
def test_plan_refusals(L, bad):
    with pytest.raises(A.AsrSpecError, match="INVAL"):
        A.asr_spec_pool_plan([array(), array(**bad)], 32)


def test_plans(L):
    assert A.asr_spec_pool_plan([array(), array(rows=2, row_slots=16, row_bytes=4, row_stride=4)], 32).nbytes >= 2 * 64
    assert A.asr_spec_pool_plan([], 32).nbytes > 0
    assert L.asr_spec_pool_plan_bytes(-1) == INVAL and L.asr_spec_pool_plan_bytes(1025) == INVAL
    buf = np.zeros(256, np.uint64)
    a = (A.AsrPageArray * 1)(array())
    assert L.asr_spec_pool_plan(a, 1, 24, buf.ctypes.data) == INVAL
    assert L.asr_spec_pool_plan(a, 1, 32, None) == INVAL
    assert L.asr_spec_pool_plan(None, 1, 32, buf.ctypes.data) == INVAL
    huge = (A.AsrPageArray * 1)(array(heads=1 << 30, page_stride=1 << 39))
    assert L.asr_spec_pool_plan(huge, 1, 32, buf.ctypes.data) == CAPACITY


@pytest.mark.parametrize("bad", [
    dict(logits=None), dict(out=None), dict(batch=0), dict(batch=65536), dict(rows=0), dict(rows=33), dict(vocab=0), dict(dtype=3),
    dict(dtype=-1), dict(logits=4098), dict(out=8193), dict(row_stride=99), dict(out_row_stride=99), dict(batch_stride=99),
    dict(out_batch_stride=0), dict(batch_stride=-400), dict(out=4096, out_row_stride=101), dict(out=4096, out_batch_stride=401),
    dict(history=None), dict(history_max=-1), dict(history_max=(1 << 30) + 1, history_stride=1 << 31), dict(history_stride=19), dict(history=66), dict(history_len=66), dict(prompt_len=65),
    dict(draft=65), dict(lens=65), dict(repetition=65), dict(frequency=65), dict(presence=65), dict(bias=65), dict(mask=66),
    dict(bias_stride=-1), dict(mask_row_stride=-1), dict(mask_batch_stride=-1), dict(repetition_all=0.0), dict(repetition_all=-1.0),
    dict(repetition_all=float("nan")), dict(frequency_all=float("inf")), dict(presence_all=float("nan")), dict(status=2), None], ids=str)
def test_rules_refusals(L, bad):
    assert L.asr_spec_adjust_logits(None if bad is None else ref(rules(**bad)), None) == INVAL


def test_tensors_must_be_on_a_gpu():
    import torch
    from paper_2608_12703_gb300 import serving
    k, s = torch.zeros(2, 2, 16, 64).to(torch.float8_e4m3fn), torch.ones(2, 2, 1)
    with pytest.raises(A.AsrSpecError, match="INVAL"):
        serving.PagedCache8(k, k, s, s, torch.zeros(1, 2, dtype=torch.int32))
    with pytest.raises(A.AsrSpecError, match="INVAL"):
        serving.adjust_logits(torch.zeros(1, 2, 8))
    with pytest.raises(A.AsrSpecError, match="INVAL"):
        serving.PagePool([], torch.zeros(1, dtype=torch.int32), torch.zeros(2, dtype=torch.int32))
