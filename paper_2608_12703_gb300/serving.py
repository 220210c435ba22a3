"""Sampled decoding over a paged K/V cache: attention over pages with the
append of new rows, accumulated attention weights, eviction down to a budget,
and acceptance of drafted tokens from given random numbers.

``PagedCache`` wraps the caller's pool of pages and page table; its methods and
``accept_sampled`` are one C-ABI call each (include/asrspec.h), on the current
CUDA stream of the tensors' device, without a synchronisation.  Outputs come
from torch's allocator; a cache keeps one workspace per stream.  Arguments are
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


class PagedCache:
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

    def _rows(self, q, kv_len, rows, k_new, v_new, causal, scale):
        B, K, D = self.batch, self.kv_heads, self.head_dim
        _need(isinstance(q, torch.Tensor) and q.dim() == 4 and q.shape[0] == B and q.shape[3] == D,
              f"q: [{B}, rows, heads, {D}] is required")
        R, H = q.shape[1], q.shape[2]
        _tensor(q, "q", self.dtype, (B, R, H, D), self.device)
        _need(R >= 1 and H >= K and H % K == 0, f"q: heads must be a multiple of the cache's {K}")
        _need(q.stride(3) == 1, "q: the last axis must be contiguous")
        _whole(kv_len, "kv_len", torch.int32, (B,), self.device)
        if rows is not None:
            _whole(rows, "rows", torch.int32, (B,), self.device)
        ns = (0, 0, 0)
        _need((k_new is None) == (v_new is None), "k_new and v_new go together")
        if k_new is not None:
            _need(causal, "k_new: rows are appended by causal calls only")
            _tensor(k_new, "k_new", self.dtype, (B, R, K, D), self.device)
            _tensor(v_new, "v_new", self.dtype, (B, R, K, D), self.device)
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
        rc = self._weigh(self._ref, _byref(r), _byref(s), lse.data_ptr(), *lse_strides, _raw_stream(self._index))
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
