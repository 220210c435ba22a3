"""Sampled decoding over a paged K/V cache: attention over pages with the
append of new rows, in 16 or 32 bits or with the cache in 8, accumulated
attention weights, eviction down to a budget, pages that sequences share, fork
and give back, penalties and masks on the logits, and acceptance of drafted
tokens from given random numbers.

``PagedCache`` and ``PagedCache8`` wrap the caller's pool of pages and page
table, ``PagePool`` the counts of who holds which; their methods,
``adjust_logits`` and ``accept_sampled`` are one C-ABI call each (include/asrspec.h), on the current
CUDA stream of the tensors' device, without a synchronisation.  Outputs come
from torch's allocator; a cache or pool keeps one workspace per stream.  Arguments are
checked here by shape, type and device; what only the device knows (lengths,
page ids, token ids) is checked by the kernels, which set the status word read
by ``PagedCache.status``.

A small call's kernels take less time than the checks of its arguments, so a
call whose tensors have the layouts (shape, strides, type, device) and whose
numbers have the values of an earlier one goes by that call's checks: these are
what the checks look at, and addresses, the only other thing, are checked by
the library.  A captured graph needs the cache object that it was captured with.
"""
from __future__ import annotations

import ctypes
import math
import operator
import threading
from typing import Optional

import torch

from . import asrspec as A

_DTYPE = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}
_MAX_LAYOUTS = 1024      # layouts remembered by one operator before it starts anew
_byref = ctypes.byref
_raw_stream = torch._C._cuda_getCurrentRawStream
_current_device = torch._C._cuda_getDevice
_capturing = torch._C._cuda_isCurrentStreamCapturing


def _need(ok: bool, what: str):
    if not ok:
        raise A.AsrSpecError("ASR_E_INVAL " + what)


def _number(x, name) -> float:
    """The value of a number, of a tensor's only element too (which waits for its device)."""
    try:
        return float(x + 0.0)
    except (TypeError, ValueError, RuntimeError, OverflowError):
        raise A.AsrSpecError(f"ASR_E_INVAL {name}: a number is required") from None


def _integer(x, name) -> int:
    try:
        return operator.index(x)
    except (TypeError, ValueError, RuntimeError, OverflowError):
        raise A.AsrSpecError(f"ASR_E_INVAL {name}: a whole number is required") from None


def _layouts(*args):
    """The layouts of a call's tensors, numbers by value.  Anything else has no place in a call and is like nothing
    remembered, so that the checks see it and refuse it."""
    return tuple([(x.shape, x.stride(), x.dtype, x.get_device()) if isinstance(x, torch.Tensor) else
                  x if x is None or isinstance(x, (int, float)) else object() for x in args])


def _remember(layouts: dict, key, value):
    if len(layouts) >= _MAX_LAYOUTS:
        layouts.clear()
    layouts[key] = value
    return value


def _tensor(x, name, dtype, shape, device):
    _need(isinstance(x, torch.Tensor) and x.device == device, f"{name}: a tensor on {device} is required")
    _need(x.dtype == dtype, f"{name}: {dtype} is required, not {x.dtype}")
    _need(tuple(x.shape) == tuple(shape), f"{name}: shape {tuple(shape)} is required, not {tuple(x.shape)}")


def _whole(x, name, dtype, shape, device):
    _tensor(x, name, dtype, shape, device)
    _need(x.is_contiguous(), f"{name}: must be contiguous")


def _check(rc, what):
    if rc < 0:
        raise A.AsrSpecError(f"{what}: {A.ERRORS.get(rc, rc)}")
    return rc


_words: dict = {}         # device index: status words made and cleared ahead, and how many are given out
_words_lock = threading.Lock()


def _status_word(device) -> torch.Tensor:
    """A status word that is clear whichever stream uses it first, without a wait for the current stream at every cache."""
    with _words_lock:
        words, at = _words.get(device.index, (None, 0))
        if words is None or at == words.numel():
            if _capturing():
                return torch.zeros(1, dtype=torch.int32, device=device)
            words, at = torch.zeros(1024, dtype=torch.int32, device=device), 0
            torch.cuda.current_stream(device).synchronize()
        _words[device.index] = (words, at + 1)
        return words[at:at + 1]


_turns: dict = {}         # (device index, stream): the lock of calls there


def _turn(index: int, stream: int):
    """Held while a call over pages launches: a call's kernels follow one another on its stream, whatever other host threads
    launch there.  What one of them leaves in the workspace is the next one's, and pages that a table names already are
    filled by the last."""
    return _turns.get((index, stream)) or _turns.setdefault((index, stream), threading.RLock())


def _expanded(x) -> bool:
    return any(n > 1 and s == 0 for n, s in zip(x.shape, x.stride()))


class _Paged:
    """What the classes over a pool of pages share: a status word, workspaces, and the rows of a call."""

    def status(self) -> int:
        """Wait for the device, then return and clear the status word."""
        torch.cuda.synchronize(self.device)
        s = int(self._status.item())
        if s:
            self._status.zero_()
            torch.cuda.current_stream(self.device).synchronize()   # before any stream's next call
        return s

    def _workspace(self, op: str, stream: int, n: int) -> torch.Tensor:
        """``n`` bytes, zero at first, that only this operator's calls on this stream use; a capture gets bytes of its
        graph's own.  The caller holds the tensor until it has launched: another host thread's larger call on the stream may
        replace it here."""
        if _capturing():
            return torch.zeros(n, dtype=torch.uint8, device=self.device)
        ws = self._ws.get((op, stream))
        if ws is None or ws.numel() < n:
            with self._lock:
                ws = self._ws.get((op, stream))
                if ws is None or ws.numel() < n:
                    ws = self._ws[(op, stream)] = torch.zeros(n, dtype=torch.uint8, device=self.device)
        return ws

    def _row_type(self, q):
        """The type that the rows of a call have."""
        return self.dtype

    def _rows(self, q, kv_len, rows, k_new, v_new, causal, scale):
        B, K, D = self.batch, self.kv_heads, self.head_dim
        dtype = self._row_type(q)
        _need(isinstance(q, torch.Tensor) and q.dim() == 4 and q.shape[0] == B and q.shape[3] == D,
              f"q: [{B}, rows, heads, {D}] is required")
        R, H = q.shape[1], q.shape[2]
        _tensor(q, "q", dtype, (B, R, H, D), self.device)
        _need(R >= 1 and H >= K and H % K == 0, f"q: heads must be a multiple of the cache's {K}")
        _need(q.stride(3) == 1, "q: the last axis must be contiguous")
        _whole(kv_len, "kv_len", torch.int32, (B,), self.device)
        if rows is not None:
            _whole(rows, "rows", torch.int32, (B,), self.device)
        ns = (0, 0, 0)
        _need((k_new is None) == (v_new is None), "k_new and v_new go together")
        if k_new is not None:
            _need(causal, "k_new: rows are appended by causal calls only")
            _tensor(k_new, "k_new", dtype, (B, R, K, D), self.device)
            _tensor(v_new, "v_new", dtype, (B, R, K, D), self.device)
            _need(k_new.stride() == v_new.stride() and k_new.stride(3) == 1,
                  "k_new and v_new: the same strides and a contiguous last axis are required")
            ns = k_new.stride()[:3]
        s = q.stride()
        return A.AsrPagedRows(q.data_ptr(), s[0], s[1], s[2], A.addr(k_new), A.addr(v_new), *ns, kv_len.data_ptr(),
                              A.addr(rows), R, H, int(causal), 1.0 / math.sqrt(D) if scale is None else scale)

    @staticmethod
    def _rows_at(layout, q, kv_len, rows, k_new, v_new):
        """The rows of an earlier call with this call's addresses."""
        r = A.AsrPagedRows.from_buffer_copy(layout)
        r.q, r.kv_len = q.data_ptr(), kv_len.data_ptr()
        if rows is not None:
            r.rows = rows.data_ptr()
        if k_new is not None:
            r.k_new, r.v_new = k_new.data_ptr(), v_new.data_ptr()
        return r


class PagedCache(_Paged):
    """A pool of K and V pages ``[n_pages, kv_heads, page_size, head_dim]`` (any strides with a
    contiguous last axis, the same for both) and the sequences' page table ``[batch, max_pages]``.

    The caller owns the three tensors and may rewrite table entries between calls.  ``status`` reads
    and clears the device status word (0 = clean, else ``asrspec.ST_*`` bits)."""

    def __init__(self, k_pages: torch.Tensor, v_pages: torch.Tensor, page_table: torch.Tensor):
        _need(isinstance(k_pages, torch.Tensor) and k_pages.is_cuda, "k_pages: a CUDA tensor is required")
        dev = k_pages.device
        _need(k_pages.dim() == 4 and k_pages.dtype in _DTYPE,
              "k_pages: [n_pages, kv_heads, page_size, head_dim] of float32, bfloat16 or float16 is required")
        _tensor(v_pages, "v_pages", k_pages.dtype, k_pages.shape, dev)
        _need(k_pages.stride() == v_pages.stride(), "k_pages and v_pages: the same strides are required")
        _need(k_pages.stride(3) == 1, "k_pages: the last axis must be contiguous")
        _need(isinstance(page_table, torch.Tensor) and page_table.device == dev and page_table.dtype == torch.int32 and
              page_table.dim() == 2 and page_table.stride(1) == 1, f"page_table: int32 [batch, max_pages] on {dev} is required")
        n_pages, kv_heads, page_size, dim = k_pages.shape
        _need(dim in (64, 128), f"head_dim 64 or 128 is required, not {dim}")
        _need(page_size >= 16 and page_size % 16 == 0, f"page_size: a multiple of 16 is required, not {page_size}")
        self.k_pages, self.v_pages, self.page_table = k_pages, v_pages, page_table
        self.device, self.dtype = dev, k_pages.dtype
        self.batch, self.max_pages = page_table.shape
        self.kv_heads, self.page_size, self.head_dim = kv_heads, page_size, dim
        self.max_slots = self.max_pages * page_size
        self._index = dev.index
        self._status = _status_word(dev)
        self._c = A.AsrPagedCache(
            k_pages.data_ptr(), v_pages.data_ptr(), k_pages.stride(0), k_pages.stride(1), k_pages.stride(2),
            page_table.data_ptr(), page_table.stride(0), n_pages, page_size, self.max_pages, kv_heads, dim, self.batch,
            _DTYPE[self.dtype], self._status.data_ptr())
        self._ref = ctypes.byref(self._c)
        self._lib = A.lib()
        self._attend, self._weigh, self._evict = (self._lib.asr_spec_paged_attend, self._lib.asr_spec_paged_weigh,
                                                  self._lib.asr_spec_paged_evict)
        self._attend_layouts, self._weigh_layouts, self._evict_layouts = {}, {}, {}
        self._ws, self._lock = {}, threading.Lock()

    def attend(self, q, kv_len, *, k_new=None, v_new=None, rows=None, causal=True, scale: Optional[float] = None,
               out=None, lse=None):
        """Attention of the block's rows ``q [B, R, H, D]`` over the cache; ``k_new`` / ``v_new`` ``[B, R, K, D]`` are
        appended at ``kv_len``.  ``rows`` (int32 ``[B]``) are the rows in use.  Causal: row i sees slots 0 .. kv_len + i;
        else slots below kv_len.  Returns ``(out [B, R, H, D], lse [B, R, H])``; ``scale`` defaults to 1 / sqrt(D)."""
        if _current_device() != self._index:
            with torch.cuda.device(self.device):
                return self.attend(q, kv_len, k_new=k_new, v_new=v_new, rows=rows, causal=causal, scale=scale, out=out,
                                   lse=lse)
        causal = bool(causal)
        if scale is not None:
            scale = _number(scale, "scale")
        key = _layouts(q, kv_len, k_new, v_new, rows, causal, scale, out, lse)
        known = self._attend_layouts.get(key)
        if known is None:
            r = self._rows(q, kv_len, rows, k_new, v_new, causal, scale)
            if out is not None:
                _whole(out, "out", self.dtype, q.shape, self.device)
            if lse is not None:
                _whole(lse, "lse", torch.float32, q.shape[:3], self.device)
            n = _check(self._lib.asr_spec_paged_attend_ws(self._ref, ctypes.byref(r)), "asr_spec_paged_attend_ws")
            known = _remember(self._attend_layouts, key, (r, n, q.shape, q.shape[:3]))
        layout, n, out_shape, lse_shape = known
        r = self._rows_at(layout, q, kv_len, rows, k_new, v_new)
        if out is None:
            out = torch.empty(out_shape, dtype=self.dtype, device=self.device)
        if lse is None:
            lse = torch.empty(lse_shape, dtype=torch.float32, device=self.device)
        stream = _raw_stream(self._index)
        ws = self._workspace("attend", stream, n)
        with _turn(self._index, stream):
            rc = self._attend(self._ref, _byref(r), out.data_ptr(), lse.data_ptr(), ws.data_ptr(), n, stream)
        if rc:
            _check(rc, "asr_spec_paged_attend")
        return out, lse

    def weigh(self, q, lse, kv_len, score, *, rows=None, causal=True, scale: Optional[float] = None, out=None, pos=None,
              first_pos=None):
        """Add the attention weight that the first ``rows`` rows gave each slot to ``score`` ``[B, K, slots]`` (fp32;
        None: zeros, then ``out`` is required).  Call it after the verification with the committed rows, and the
        ``kv_len`` and ``lse`` of the attention.  Writes ``out`` (default: ``score`` in place) and, with ``pos`` (int32,
        as score) and ``first_pos`` (int32 ``[B]``), the new slots' positions.  Returns ``out``."""
        if _current_device() != self._index:
            with torch.cuda.device(self.device):
                return self.weigh(q, lse, kv_len, score, rows=rows, causal=causal, scale=scale, out=out, pos=pos,
                                  first_pos=first_pos)
        out = score if out is None else out
        causal = bool(causal)
        if scale is not None:
            scale = _number(scale, "scale")
        key = _layouts(q, kv_len, rows, causal, scale, lse, score, out, pos, first_pos)
        known = self._weigh_layouts.get(key)
        if known is None:
            known = _remember(self._weigh_layouts, key, self._weigh_layout(q, lse, kv_len, score, rows, causal, scale, out,
                                                                           pos, first_pos))
        layout, slots, lse_strides = known
        r = self._rows_at(layout, q, kv_len, rows, None, None)
        s = A.AsrPagedScores.from_buffer_copy(slots)
        s.score_out = out.data_ptr()
        if score is not None:
            s.score = score.data_ptr()
        if pos is not None:
            s.pos, s.first_pos = pos.data_ptr(), first_pos.data_ptr()
        stream = _raw_stream(self._index)
        with _turn(self._index, stream):
            rc = self._weigh(self._ref, _byref(r), _byref(s), lse.data_ptr(), *lse_strides, stream)
        if rc:
            _check(rc, "asr_spec_paged_weigh")
        return out

    def _weigh_layout(self, q, lse, kv_len, score, rows, causal, scale, out, pos, first_pos):
        r = self._rows(q, kv_len, rows, None, None, causal, scale)
        B, R, H = q.shape[:3]
        _need(out is not None, "out: required without score")
        _need(isinstance(out, torch.Tensor) and out.dim() == 3, "score: [batch, kv_heads, slots] is required")
        shape = (B, self.kv_heads, out.shape[2])
        _tensor(out, "out", torch.float32, shape, self.device)
        _need(out.stride(2) == 1, "out: the last axis must be contiguous")
        for x, name, dt in ((score, "score", torch.float32), (pos, "pos", torch.int32)):
            if x is not None:
                _tensor(x, name, dt, shape, self.device)
                _need(x.stride() == out.stride(), f"{name}: out's strides are required")
        _need((pos is None) == (first_pos is None), "pos and first_pos go together")
        if first_pos is not None:
            _whole(first_pos, "first_pos", torch.int32, (B,), self.device)
        _tensor(lse, "lse", torch.float32, (B, R, H), self.device)
        _need(lse.stride(2) == 1, "lse: the last axis must be contiguous")
        s = A.AsrPagedScores(None, None, out.stride(0), out.stride(1), shape[2], None, None, 0, 0, 0, None)
        return r, s, (lse.stride(0), lse.stride(1))

    def evict(self, lens, score, pos, seen, *, budget: int, recent: int = 0, first: int = 0, lens_out=None, score_out=None,
              pos_out=None):
        """Cut every head to its ``budget`` slots of highest accumulated weight; the ``recent`` newest positions
        (of ``seen`` ``[B]`` tokens) and the ``first`` oldest go last (of more than the budget holds the lowest slots stay,
        whatever their scores).  Freed slots below the budget take the kept ones
        past it.  ``score`` / ``pos`` ``[B, K, slots]`` and the pages' K/V move along: into ``score_out`` / ``pos_out``
        (default: in place) and in place.  Returns ``(lens_out, score_out, pos_out)``."""
        if _current_device() != self._index:
            with torch.cuda.device(self.device):
                return self.evict(lens, score, pos, seen, budget=budget, recent=recent, first=first, lens_out=lens_out,
                                  score_out=score_out, pos_out=pos_out)
        score_out = score if score_out is None else score_out
        pos_out = pos if pos_out is None else pos_out
        budget, recent, first = _integer(budget, "budget"), _integer(recent, "recent"), _integer(first, "first")
        key = _layouts(lens, score, pos, seen, budget, recent, first, lens_out, score_out, pos_out)
        known = self._evict_layouts.get(key)
        if known is None:
            known = _remember(self._evict_layouts, key, self._evict_layout(lens, score, pos, seen, budget, recent, first,
                                                                           lens_out, score_out, pos_out))
        slots, n = known
        if lens_out is None:
            lens_out = torch.empty_like(lens)
        s = A.AsrPagedScores.from_buffer_copy(slots)
        s.score, s.pos, s.score_out, s.pos_out = score.data_ptr(), pos.data_ptr(), score_out.data_ptr(), pos_out.data_ptr()
        stream = _raw_stream(self._index)
        ws = self._workspace("evict", stream, n)
        with _turn(self._index, stream):
            rc = self._evict(self._ref, _byref(s), lens.data_ptr(), seen.data_ptr(), budget, recent, first, lens_out.data_ptr(),
                             ws.data_ptr(), n, stream)
        if rc:
            _check(rc, "asr_spec_paged_evict")
        return lens_out, score_out, pos_out

    def _evict_layout(self, lens, score, pos, seen, budget, recent, first, lens_out, score_out, pos_out):
        B, K = self.batch, self.kv_heads
        _whole(lens, "lens", torch.int32, (B,), self.device)
        _whole(seen, "seen", torch.int32, (B,), self.device)
        if lens_out is not None:
            _whole(lens_out, "lens_out", torch.int32, (B,), self.device)
        for x, y, name in ((score, pos, "score"), (score_out, pos_out, "score_out")):
            _need(isinstance(x, torch.Tensor) and x.dim() == 3, f"{name}: [batch, kv_heads, slots] is required")
            _tensor(x, name, torch.float32, (B, K, x.shape[2]), self.device)
            _tensor(y, name.replace("score", "pos"), torch.int32, x.shape, self.device)
            _need(x.stride() == y.stride() and x.stride(2) == 1,
                  "score and pos: the same strides and a contiguous last axis are required")
        _need(budget >= 1 and recent >= 0 and first >= 0, "budget >= 1, recent >= 0 and first >= 0 are required")
        _need(max(budget, recent, first) < 1 << 31, "budget, recent and first: at most 2^31 - 1")
        s = A.AsrPagedScores(None, None, score.stride(0), score.stride(1), score.shape[2], None, None, score_out.stride(0),
                             score_out.stride(1), score_out.shape[2], None)
        n = _check(self._lib.asr_spec_paged_evict_ws(self._ref, ctypes.byref(s), budget), "asr_spec_paged_evict_ws")
        return s, n


class PagedCache8(_Paged):
    """A pool of pages held in 8 bits: codes ``[n_pages, kv_heads, page_size, head_dim]`` (float8_e4m3fn, any strides with a
    contiguous last axis, the same for both), scales ``[n_pages, kv_heads, page_size / 16]`` (float32, positive, the same
    strides for both), one for the 16 slots of a group and a head, and the page table ``[batch, max_pages]``.

    A slot's values are its codes times its group's scale.  The caller owns the tensors.  The scales of appended groups are
    powers of two; those of groups that were filled in another way need not be.  Scales that share memory (one expanded over
    pages or heads, the same ones for K and V) can be read but not appended under."""

    def __init__(self, k_pages: torch.Tensor, v_pages: torch.Tensor, k_scale: torch.Tensor, v_scale: torch.Tensor,
                 page_table: torch.Tensor):
        _need(isinstance(k_pages, torch.Tensor) and k_pages.is_cuda, "k_pages: a CUDA tensor is required")
        dev = k_pages.device
        _need(k_pages.dim() == 4 and k_pages.dtype == torch.float8_e4m3fn,
              "k_pages: [n_pages, kv_heads, page_size, head_dim] of float8_e4m3fn is required")
        _tensor(v_pages, "v_pages", k_pages.dtype, k_pages.shape, dev)
        _need(k_pages.stride() == v_pages.stride(), "k_pages and v_pages: the same strides are required")
        _need(k_pages.stride(3) == 1, "k_pages: the last axis must be contiguous")
        _need(isinstance(page_table, torch.Tensor) and page_table.device == dev and page_table.dtype == torch.int32 and
              page_table.dim() == 2 and page_table.stride(1) == 1, f"page_table: int32 [batch, max_pages] on {dev} is required")
        n_pages, kv_heads, page_size, dim = k_pages.shape
        _need(dim in (64, 128), f"head_dim 64 or 128 is required, not {dim}")
        _need(page_size >= 16 and page_size % 16 == 0, f"page_size: a multiple of 16 is required, not {page_size}")
        for x, name in ((k_scale, "k_scale"), (v_scale, "v_scale")):
            _tensor(x, name, torch.float32, (n_pages, kv_heads, page_size // 16), dev)
            _need(x.stride(2) == 1 or page_size == 16, f"{name}: the last axis must be contiguous")
        _need(k_scale.stride()[:2] == v_scale.stride()[:2], "k_scale and v_scale: the same strides are required")
        self.k_pages, self.v_pages, self.k_scale, self.v_scale, self.page_table = k_pages, v_pages, k_scale, v_scale, page_table
        self.device = dev
        self.batch, self.max_pages = page_table.shape
        self.kv_heads, self.page_size, self.head_dim = kv_heads, page_size, dim
        self.max_slots = self.max_pages * page_size
        self._index = dev.index
        self._status = _status_word(dev)
        self._c = A.AsrPaged8Cache(
            k_pages.data_ptr(), v_pages.data_ptr(), k_pages.stride(0), k_pages.stride(1), k_pages.stride(2),
            k_scale.data_ptr(), v_scale.data_ptr(), k_scale.stride(0), k_scale.stride(1), page_table.data_ptr(),
            page_table.stride(0), n_pages, page_size, self.max_pages, kv_heads, dim, self.batch, self._status.data_ptr())
        self._ref = ctypes.byref(self._c)
        self._lib = A.lib()
        self._attend, self._append = self._lib.asr_spec_paged8_attend, self._lib.asr_spec_paged8_append
        self._attend_layouts, self._append_layouts = {}, {}
        self._ws, self._lock = {}, threading.Lock()
        self._read_only = (k_scale.data_ptr() == v_scale.data_ptr() or k_pages.data_ptr() == v_pages.data_ptr() or
                           _expanded(k_scale))

    def _need_own(self):
        _need(not self._read_only, "k_new: appended rows need codes and scales of their own; those that K and V, pages or heads "
                                   "share can only be read")

    def _row_type(self, q):
        dtype = getattr(q, "dtype", None)
        _need(dtype in (torch.bfloat16, torch.float16), f"q: bfloat16 or float16 is required, not {dtype}")
        return dtype

    def append(self, k_new, v_new, kv_len, *, rows=None):
        """Quantise ``k_new`` / ``v_new`` ``[B, R, K, D]`` (float32, bfloat16 or float16) behind each sequence's ``kv_len``
        slots; ``rows`` (int32 ``[B]``) are the rows in use.  A group that the rows begin takes the least power of two that
        holds its values; one that goes on keeps its scale, or takes a larger one and its codes are rounded anew.  Rows that are
        rejected later leave the scale that they raised (see ``asr_spec_paged8_append``)."""
        if _current_device() != self._index:
            with torch.cuda.device(self.device):
                return self.append(k_new, v_new, kv_len, rows=rows)
        key = _layouts(k_new, v_new, kv_len, rows)
        known = self._append_layouts.get(key)
        if known is None:
            self._need_own()
            B, K, D = self.batch, self.kv_heads, self.head_dim
            _need(isinstance(k_new, torch.Tensor) and k_new.dim() == 4 and k_new.dtype in _DTYPE and k_new.shape[1] >= 1,
                  f"k_new: [{B}, rows, {K}, {D}] of float32, bfloat16 or float16 is required")
            shape = (B, k_new.shape[1], K, D)
            _tensor(k_new, "k_new", k_new.dtype, shape, self.device)
            _tensor(v_new, "v_new", k_new.dtype, shape, self.device)
            _need(k_new.stride() == v_new.stride() and k_new.stride(3) == 1,
                  "k_new and v_new: the same strides and a contiguous last axis are required")
            _whole(kv_len, "kv_len", torch.int32, (B,), self.device)
            if rows is not None:
                _whole(rows, "rows", torch.int32, (B,), self.device)
            s = k_new.stride()
            known = _remember(self._append_layouts, key, (
                A.AsrPagedRows(None, 0, 0, 0, k_new.data_ptr(), v_new.data_ptr(), s[0], s[1], s[2], kv_len.data_ptr(),
                               A.addr(rows), shape[1], K, 1, 1.0), _DTYPE[k_new.dtype]))
        layout, dtype = known
        r = A.AsrPagedRows.from_buffer_copy(layout)
        r.k_new, r.v_new, r.kv_len = k_new.data_ptr(), v_new.data_ptr(), kv_len.data_ptr()
        if rows is not None:
            r.rows = rows.data_ptr()
        stream = _raw_stream(self._index)
        with _turn(self._index, stream):
            rc = self._append(self._ref, _byref(r), dtype, stream)
        if rc:
            _check(rc, "asr_spec_paged8_append")

    def attend(self, q, kv_len, *, k_new=None, v_new=None, rows=None, causal=True, scale: Optional[float] = None,
               out=None, lse=None):
        """As ``PagedCache.attend``, for ``q``, ``k_new`` and ``v_new`` in bfloat16 or float16.  New rows are appended as by
        ``append`` and seen as they are stored."""
        if _current_device() != self._index:
            with torch.cuda.device(self.device):
                return self.attend(q, kv_len, k_new=k_new, v_new=v_new, rows=rows, causal=causal, scale=scale, out=out,
                                   lse=lse)
        causal = bool(causal)
        if scale is not None:
            scale = _number(scale, "scale")
        key = _layouts(q, kv_len, k_new, v_new, rows, causal, scale, out, lse)
        known = self._attend_layouts.get(key)
        if known is None:
            r = self._rows(q, kv_len, rows, k_new, v_new, causal, scale)
            if k_new is not None:
                self._need_own()
            if out is not None:
                _whole(out, "out", q.dtype, q.shape, self.device)
            if lse is not None:
                _whole(lse, "lse", torch.float32, q.shape[:3], self.device)
            dtype = _DTYPE[q.dtype]
            n = _check(self._lib.asr_spec_paged8_attend_ws(self._ref, ctypes.byref(r), dtype), "asr_spec_paged8_attend_ws")
            known = _remember(self._attend_layouts, key, (r, n, q.shape, q.shape[:3], dtype))
        layout, n, out_shape, lse_shape, dtype = known
        r = self._rows_at(layout, q, kv_len, rows, k_new, v_new)
        if out is None:
            out = torch.empty(out_shape, dtype=q.dtype, device=self.device)
        if lse is None:
            lse = torch.empty(lse_shape, dtype=torch.float32, device=self.device)
        stream = _raw_stream(self._index)
        ws = self._workspace("attend", stream, n)
        with _turn(self._index, stream):
            rc = self._attend(self._ref, _byref(r), dtype, out.data_ptr(), lse.data_ptr(), ws.data_ptr(), n, stream)
        if rc:
            _check(rc, "asr_spec_paged8_attend")
        return out, lse


class PagePool(_Paged):
    """Who holds which pages of one or more caches (one a layer) that share a page table: ``held [batch]``, the entries in
    use of each table row, and ``refs [n_pages]``, how many table entries (and holders of the caller's own) a page has; 0 is
    free.  Both int32, contiguous.

    A page that several rows hold may be read by all and written by none: ``reserve`` comes before an append, and
    ``PagedCache.evict``, which moves slots within their pages, only where no page is shared.

    The calls decide from these arrays alone and keep nothing: each takes the lowest free pages in order of sequence and
    slot.  They write the caches' table, ``held`` and ``refs`` in place unless outputs are given (which take all of the new
    state; table entries at or past a row's held ones are left as they are)."""

    def __init__(self, caches, held: torch.Tensor, refs: torch.Tensor):
        caches = list(caches) if isinstance(caches, (list, tuple)) else [caches]
        _need(len(caches) > 0 and all(isinstance(c, (PagedCache, PagedCache8)) for c in caches),
              "caches: PagedCache or PagedCache8 objects are required")
        c0 = caches[0]
        table, n_pages = c0.page_table, c0.k_pages.shape[0]
        for c in caches:
            t = c.page_table
            _need(t.data_ptr() == table.data_ptr() and t.shape == table.shape and t.stride() == table.stride() and
                  c.device == c0.device, "caches: the same page table is required")
            _need(c.k_pages.shape[0] == n_pages and c.page_size == c0.page_size,
                  "caches: the same number and size of pages are required")
            if isinstance(c, PagedCache8):
                _need(not _expanded(c.k_scale), "caches: pages need scales of their own; those that pages or heads share cannot be moved")
        _whole(held, "held", torch.int32, (c0.batch,), c0.device)
        _whole(refs, "refs", torch.int32, (n_pages,), c0.device)
        _need(not _capturing(), "a pool is made outside of a graph capture")
        self.caches, self.page_table, self.held, self.refs = caches, table, held, refs
        self.device, self.batch, self.max_pages, self.page_size = c0.device, c0.batch, c0.max_pages, c0.page_size
        self.n_pages, self._index = n_pages, c0.device.index
        arrays = []
        for c in caches:
            for x in (c.k_pages, c.v_pages):
                es = x.element_size()
                arrays.append(A.AsrPageArray(x.data_ptr(), x.stride(0) * es, x.stride(1) * es, x.stride(2) * es, c.kv_heads,
                                             c.page_size, c.head_dim * es, 1))
            if isinstance(c, PagedCache8):
                for x in (c.k_scale, c.v_scale):
                    arrays.append(A.AsrPageArray(x.data_ptr(), x.stride(0) * 4, x.stride(1) * 4, 4, c.kv_heads,
                                                 c.page_size // 16, 4, 16))
        _need(len(arrays) <= 1024, "caches: at most 1024 arrays (keys, values, scales of every layer)")
        with torch.cuda.device(self.device):
            self._status = _status_word(self.device)
            self._plan = torch.from_numpy(A.asr_spec_pool_plan(arrays, self.page_size)).to(self.device)
            torch.cuda.current_stream().synchronize()   # before any stream's call
        self._n = len(arrays)
        self._lib = A.lib()
        s = table.stride(0)
        self._layout = A.AsrPagePool(table.data_ptr(), s, held.data_ptr(), refs.data_ptr(), table.data_ptr(), s, held.data_ptr(),
                                     refs.data_ptr(), n_pages, self.page_size, self.max_pages, self.batch,
                                     self._status.data_ptr())
        self._bytes = _check(self._lib.asr_spec_pool_ws(ctypes.byref(self._layout)), "asr_spec_pool_ws")
        self._reserve, self._fork, self._compact = (self._lib.asr_spec_pool_reserve, self._lib.asr_spec_pool_fork,
                                                    self._lib.asr_spec_pool_compact)
        self._layouts, self._ws, self._lock = {}, {}, threading.Lock()

    def _checked(self, key, names, ints, table_out, held_out, refs_out):
        """Checks of a call's arguments, once a layout: ``ints`` are [batch]."""
        for x, name in zip(ints, names):
            if x is not None:
                _whole(x, name, torch.int32, (self.batch,), self.device)
        layout = A.AsrPagePool.from_buffer_copy(self._layout)
        if table_out is not None:
            _tensor(table_out, "table_out", torch.int32, (self.batch, self.max_pages), self.device)
            _need(table_out.stride(1) == 1 or self.max_pages == 1, "table_out: the last axis must be contiguous")
            layout.table_out_stride = max(table_out.stride(0), self.max_pages) if self.batch == 1 else table_out.stride(0)
        if held_out is not None:
            _whole(held_out, "held_out", torch.int32, (self.batch,), self.device)
        if refs_out is not None:
            _whole(refs_out, "refs_out", torch.int32, (self.n_pages,), self.device)
        return _remember(self._layouts, key, layout)

    @staticmethod
    def _at(layout, table_out, held_out, refs_out):
        """The pool of an earlier call with this call's outputs."""
        p = A.AsrPagePool.from_buffer_copy(layout)
        if table_out is not None:
            p.table_out = table_out.data_ptr()
        if held_out is not None:
            p.held_out = held_out.data_ptr()
        if refs_out is not None:
            p.refs_out = refs_out.data_ptr()
        return p

    def reserve(self, lens, rows, *, table_out=None, held_out=None, refs_out=None):
        """Private pages for ``rows [B]`` slots behind ``lens [B]`` of each sequence: missing pages are taken from the pool,
        and one that others hold too is replaced by a copy of its slots below ``lens`` in every cache; of sequences that
        alone share the page of slot ``lens`` the lowest keeps it.  A pool with too few free pages leaves everything as it
        is (``ST_CAPACITY``).  Returns ``(table, held, refs, counts)``, counts (on the device) being the pages taken and
        those free afterwards."""
        if _current_device() != self._index:
            with torch.cuda.device(self.device):
                return self.reserve(lens, rows, table_out=table_out, held_out=held_out, refs_out=refs_out)
        _need(lens is not None and rows is not None, "lens and rows are required")
        key = (0, _layouts(lens, rows, table_out, held_out, refs_out))
        layout = self._layouts.get(key) or self._checked(key, ("lens", "rows"), (lens, rows), table_out, held_out, refs_out)
        p = self._at(layout, table_out, held_out, refs_out)
        counts = torch.empty(2, dtype=torch.int32, device=self.device)
        stream = _raw_stream(self._index)
        ws = self._workspace("pool", stream, self._bytes)
        with _turn(self._index, stream):
            rc = self._reserve(_byref(p), self._plan.data_ptr(), self._n, lens.data_ptr(), rows.data_ptr(), counts.data_ptr(),
                               ws.data_ptr(), self._bytes, stream)
        if rc:
            _check(rc, "asr_spec_pool_reserve")
        return (self.page_table if table_out is None else table_out, self.held if held_out is None else held_out,
                self.refs if refs_out is None else refs_out, counts)

    def fork(self, parent=None, keep=None, *, table_out=None, held_out=None, refs_out=None):
        """Sequence b goes on with the pages of sequence ``parent[b]`` as they were before the call (None: its own; -1:
        none), of which it holds those of the first ``keep[b]`` slots (None: all).  Nothing is copied: shared pages are
        copied by ``reserve`` when they are about to be written.  Returns ``(table, held, refs)``."""
        if _current_device() != self._index:
            with torch.cuda.device(self.device):
                return self.fork(parent, keep, table_out=table_out, held_out=held_out, refs_out=refs_out)
        key = (1, _layouts(parent, keep, table_out, held_out, refs_out))
        layout = self._layouts.get(key) or self._checked(key, ("parent", "keep"), (parent, keep), table_out, held_out, refs_out)
        p = self._at(layout, table_out, held_out, refs_out)
        stream = _raw_stream(self._index)
        ws = self._workspace("pool", stream, self._bytes)
        with _turn(self._index, stream):
            rc = self._fork(_byref(p), None if parent is None else parent.data_ptr(), None if keep is None else keep.data_ptr(),
                            ws.data_ptr(), self._bytes, stream)
        if rc:
            _check(rc, "asr_spec_pool_fork")
        return (self.page_table if table_out is None else table_out, self.held if held_out is None else held_out,
                self.refs if refs_out is None else refs_out)

    def compact(self, *, table_out=None, refs_out=None):
        """Live pages to the front of the pool: with n of them the j-th free page below n takes the contents of the j-th live
        one at or past it, in every cache, and table entries and counts follow.  Returns ``(table, refs, where, live)``:
        each page's new id (-1 for a free one) and n, on the device."""
        if _current_device() != self._index:
            with torch.cuda.device(self.device):
                return self.compact(table_out=table_out, refs_out=refs_out)
        key = (2, _layouts(table_out, refs_out))
        layout = self._layouts.get(key) or self._checked(key, (), (), table_out, None, refs_out)
        p = self._at(layout, table_out, None, refs_out)
        where = torch.empty(self.n_pages, dtype=torch.int32, device=self.device)
        live = torch.empty(1, dtype=torch.int32, device=self.device)
        stream = _raw_stream(self._index)
        ws = self._workspace("pool", stream, self._bytes)
        with _turn(self._index, stream):
            rc = self._compact(_byref(p), self._plan.data_ptr(), self._n, where.data_ptr(), live.data_ptr(), ws.data_ptr(),
                               self._bytes, stream)
        if rc:
            _check(rc, "asr_spec_pool_compact")
        return (self.page_table if table_out is None else table_out, self.refs if refs_out is None else refs_out, where, live)


_adjust_layouts: dict = {}


def adjust_logits(logits, *, history=None, history_len=None, prompt_len=None, draft=None, lens=None, repetition=1.0,
                  frequency=0.0, presence=0.0, bias=None, mask=None, out=None, status=None):
    """Penalties for repeated tokens, biases and grammar masks on the logits of a block, before ``accept_sampled``.

    ``logits [B, k + 1, V]`` (float32, bfloat16 or float16); row i comes after the utterance's ``history [B, T]`` (the first
    ``history_len [B]`` of it, of which the first ``prompt_len [B]`` belong to the prompt) and its first i drafts
    (``draft [B, k]``; ``lens [B]``, -1 sits out; None: k each); tokens and lengths are int32.  With c(j) the count of token
    j among these without the prompt:  a token that occurs at all has its logit divided by ``repetition`` (multiplied if
    not positive); then ``frequency * c + presence * (c > 0)`` is subtracted, ``bias`` (float32 ``[V]`` or ``[B, V]``)
    added, and a token whose bit in ``mask`` (int32 ``[B, k + 1, ceil(V / 32)]``, bit j % 32 of word j // 32) is not set
    gets -inf.  ``repetition``, ``frequency`` and ``presence`` are numbers or float32 ``[B]``.  Writes ``out`` (default:
    ``logits`` in place) and returns it; rows past ``lens`` are left as they are."""
    if not (type(repetition) is float or isinstance(repetition, torch.Tensor) and repetition.dim() == 1):
        repetition = _number(repetition, "repetition")
    if not (type(frequency) is float or isinstance(frequency, torch.Tensor) and frequency.dim() == 1):
        frequency = _number(frequency, "frequency")
    if not (type(presence) is float or isinstance(presence, torch.Tensor) and presence.dim() == 1):
        presence = _number(presence, "presence")
    key = _layouts(logits, history, history_len, prompt_len, draft, lens, repetition, frequency, presence, bias, mask, out, status)
    known = _adjust_layouts.get(key)
    if known is None:
        known = _remember(_adjust_layouts, key, _adjust_layout(logits, history, history_len, prompt_len, draft, lens, repetition,
                                                               frequency, presence, bias, mask, out, status))
    layout, device, index, names = known
    if _current_device() != index:
        with torch.cuda.device(device):
            return adjust_logits(logits, history=history, history_len=history_len, prompt_len=prompt_len, draft=draft, lens=lens,
                                 repetition=repetition, frequency=frequency, presence=presence, bias=bias, mask=mask, out=out,
                                 status=status)
    out = logits if out is None else out
    r = A.AsrLogitRules.from_buffer_copy(layout)
    r.logits, r.out = logits.data_ptr(), out.data_ptr()
    given = (history, history_len, prompt_len, draft, lens, repetition, frequency, presence, bias, mask, status)
    for i, name in names:
        setattr(r, name, given[i].data_ptr())
    rc = _adjust(_byref(r), _raw_stream(index))
    if rc:
        _check(rc, "asr_spec_adjust_logits")
    return out


def _adjust(*args):
    """The library's entry; looked up at the first call, which loads the library."""
    global _adjust
    _adjust = A.lib().asr_spec_adjust_logits
    return _adjust(*args)


def _adjust_layout(logits, history, history_len, prompt_len, draft, lens, repetition, frequency, presence, bias, mask, out, status):
    _need(isinstance(logits, torch.Tensor) and logits.is_cuda and logits.dim() == 3 and logits.dtype in _DTYPE,
          "logits: [batch, k + 1, vocab] of float32, bfloat16 or float16 on a CUDA device is required")
    dev = logits.device
    B, R, V = logits.shape
    _need(B >= 1 and 1 <= R <= 32 and V >= 1, "logits: 1 to 32 rows are required")
    out = logits if out is None else out
    _tensor(out, "out", logits.dtype, logits.shape, dev)
    for x, name in ((logits, "logits"), (out, "out")):
        _need(x.stride(2) == 1 or V == 1, f"{name}: the last axis must be contiguous")
    if history is not None:
        _need(isinstance(history, torch.Tensor) and history.dim() == 2, f"history: int32 [{B}, tokens] is required")
        _tensor(history, "history", torch.int32, (B, history.shape[1]), dev)
        _need(history.stride(1) == 1 or history.shape[1] <= 1, "history: the last axis must be contiguous")
        _need(history.stride(0) >= history.shape[1], "history: rows must lie apart (an expanded history: contiguous() first)")
    _need(history is not None or (history_len is None and prompt_len is None), "history_len, prompt_len: history is required")
    for x, name in ((history_len, "history_len"), (prompt_len, "prompt_len"), (lens, "lens")):
        if x is not None:
            _whole(x, name, torch.int32, (B,), dev)
    if draft is not None:
        _whole(draft, "draft", torch.int32, (B, R - 1), dev)
    numbers = []
    for x, name, neutral in ((repetition, "repetition", 1.0), (frequency, "frequency", 0.0), (presence, "presence", 0.0)):
        if isinstance(x, torch.Tensor):
            _whole(x, name, torch.float32, (B,), dev)
            x = neutral
        _need(math.isfinite(x) and (name != "repetition" or x > 0), f"{name}: {x} is out of range")
        numbers.append(x)
    bias_stride = 0
    if bias is not None:
        _need(isinstance(bias, torch.Tensor) and bias.dim() in (1, 2), f"bias: float32 [{V}] or [{B}, {V}] is required")
        _tensor(bias, "bias", torch.float32, (V,) if bias.dim() == 1 else (B, V), dev)
        _need(bias.stride(-1) == 1 or V == 1, "bias: the last axis must be contiguous")
        bias_stride = bias.stride(0) if bias.dim() == 2 else 0
    mask_strides = (0, 0)
    if mask is not None:
        _tensor(mask, "mask", torch.int32, (B, R, (V + 31) // 32), dev)
        _need(mask.stride(2) == 1 or V <= 32, "mask: the last axis must be contiguous")
        mask_strides = mask.stride()[:2]
    if status is not None:
        _whole(status, "status", torch.int32, (1,), dev)
    r = A.AsrLogitRules(None, logits.stride(0), logits.stride(1), None, out.stride(0), out.stride(1), B, R, V,
                        _DTYPE[logits.dtype], None, 0 if history is None else history.stride(0),
                        0 if history is None else history.shape[1], *[None] * 7, *numbers, None, bias_stride, None, *mask_strides,
                        None)
    given = ((history, "history"), (history_len, "history_len"), (prompt_len, "prompt_len"), (draft, "draft"), (lens, "lens"),
             (repetition, "repetition"), (frequency, "frequency"), (presence, "presence"), (bias, "bias"), (mask, "mask"),
             (status, "status"))
    return r, dev, dev.index, [(i, name) for i, (x, name) in enumerate(given) if isinstance(x, torch.Tensor) and x.numel() > 0]


_accept_layouts: dict = {}


def accept_sampled(target, draft, lens, u, race, *, draft_logits=None, temperature: float = 1.0, status=None):
    """Accept drafted tokens against the target's probabilities from given random numbers.

    ``target [B, k + 1, V]`` and ``draft_logits [B, k, V]`` (None: greedy drafts) are logits of one type (float32,
    bfloat16, float16); ``draft [B, k]`` and ``lens [B]`` (-1 sits out; None: k each) are int32; ``u [B, k]`` uniform in
    [0, 1) and ``race [B, V]`` standard exponential, float32.  Returns ``(accepted [B], token [B], step [B], prob [B, k])``:
    the drafts accepted, the token drawn after them, the positions to commit and each draft's acceptance probability.
    ``status``: an int32 device tensor that collects ``asrspec.ST_*`` bits."""
    temperature = _number(temperature, "temperature")
    key = _layouts(target, draft, lens, u, race, draft_logits, status, temperature)
    known = _accept_layouts.get(key)
    if known is None:
        known = _remember(_accept_layouts, key, _accept_layout(target, draft, lens, u, race, draft_logits, temperature, status))
    layout, device, index, race_stride = known
    if _current_device() != index:
        with torch.cuda.device(device):
            return accept_sampled(target, draft, lens, u, race, draft_logits=draft_logits, temperature=temperature, status=status)
    x = A.AsrSampledLogits.from_buffer_copy(layout)
    x.target = target.data_ptr()
    if draft_logits is not None and x.k:
        x.draft_logits = draft_logits.data_ptr()
    accepted = torch.empty(x.batch, dtype=torch.int32, device=device)
    token, step, prob = torch.empty_like(accepted), torch.empty_like(accepted), torch.empty_like(u)
    rc = _accept(
        _byref(x), draft.data_ptr(), None if lens is None else lens.data_ptr(), u.data_ptr(), race.data_ptr(), race_stride,
        temperature, accepted.data_ptr(), token.data_ptr(), step.data_ptr(), prob.data_ptr(),
        None if status is None else status.data_ptr(), _raw_stream(index))
    if rc:
        _check(rc, "asr_spec_accept_sampled")
    return accepted, token, step, prob


def _accept(*args):
    """The library's entry; looked up at the first call, which loads the library."""
    global _accept
    _accept = A.lib().asr_spec_accept_sampled
    return _accept(*args)


def _accept_layout(target, draft, lens, u, race, draft_logits, temperature, status):
    _need(isinstance(target, torch.Tensor) and target.is_cuda and target.dim() == 3 and target.dtype in _DTYPE,
          "target: [batch, k + 1, vocab] of float32, bfloat16 or float16 on a CUDA device is required")
    dev = target.device
    B, k, V = target.shape[0], target.shape[1] - 1, target.shape[2]
    _need(0 <= k <= 31 and B >= 1 and V >= 1, "target: 1 to 32 rows are required")
    _need(target.stride(2) == 1, "target: the last axis must be contiguous")
    _whole(draft, "draft", torch.int32, (B, k), dev)
    if lens is not None:
        _whole(lens, "lens", torch.int32, (B,), dev)
    _whole(u, "u", torch.float32, (B, k), dev)
    _tensor(race, "race", torch.float32, (B, V), dev)
    _need(race.stride(1) == 1, "race: the last axis must be contiguous")
    ds = (0, 0)
    if draft_logits is not None:
        _tensor(draft_logits, "draft_logits", target.dtype, (B, k, V), dev)
        _need(k == 0 or draft_logits.stride(2) == 1, "draft_logits: the last axis must be contiguous")
        ds = draft_logits.stride()[:2]
    if status is not None:
        _whole(status, "status", torch.int32, (1,), dev)
    _need(temperature > 0 and math.isfinite(temperature), "temperature: a positive number is required")
    return (A.AsrSampledLogits(None, target.stride(0), target.stride(1), None, *ds, B, k, V, _DTYPE[target.dtype]), dev,
            dev.index, race.stride(0))
