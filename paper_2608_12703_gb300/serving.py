"""Sampled decoding over a paged K/V cache: attention over pages with the
append of new rows, accumulated attention weights, eviction down to a budget,
and acceptance of drafted tokens from given random numbers.

``PagedCache`` wraps the caller's pool of pages and page table; its methods and
``accept_sampled`` are one C-ABI call each (include/asrspec.h), on the current
CUDA stream of the tensors' device, without a synchronisation.  Workspaces and
outputs come from torch's allocator on that stream.  Arguments are checked
here by shape, type and device; what only the device knows (lengths, page ids,
token ids) is checked by the kernels, which set the status word read by
``PagedCache.status``.
"""
from __future__ import annotations

import ctypes
import math
from typing import Optional

import torch

from . import asrspec as A

_DTYPE = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}


def _need(ok: bool, what: str):
    if not ok:
        raise A.AsrSpecError("ASR_E_INVAL " + what)


def _tensor(x, name, dtype, shape, device):
    _need(isinstance(x, torch.Tensor) and x.device == device, f"{name}: a tensor on {device} is required")
    _need(x.dtype == dtype, f"{name}: {dtype} is required, not {x.dtype}")
    _need(tuple(x.shape) == tuple(shape), f"{name}: shape {tuple(shape)} is required, not {tuple(x.shape)}")


def _ints(x, name, shape, device):
    _tensor(x, name, torch.int32, shape, device)
    _need(x.is_contiguous(), f"{name}: must be contiguous")


def _check(rc, what):
    if rc < 0:
        raise A.AsrSpecError(f"{what}: {A.ERRORS.get(rc, rc)}")
    return rc


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
        self._status = torch.zeros(1, dtype=torch.int32, device=dev)
        self._c = A.AsrPagedCache(
            k_pages.data_ptr(), v_pages.data_ptr(), k_pages.stride(0), k_pages.stride(1), k_pages.stride(2),
            page_table.data_ptr(), page_table.stride(0), n_pages, page_size, self.max_pages, kv_heads, dim, self.batch,
            _DTYPE[self.dtype], self._status.data_ptr())
        self._ref = ctypes.byref(self._c)
        self._ws = {}

    def status(self) -> int:
        """Wait for the device, then return and clear the status word."""
        torch.cuda.synchronize(self.device)
        s = int(self._status.item())
        if s:
            self._status.zero_()
        return s

    def _rows(self, q, kv_len, rows, k_new, v_new, causal, scale):
        B, K, D = self.batch, self.kv_heads, self.head_dim
        _need(isinstance(q, torch.Tensor) and q.dim() == 4 and q.shape[0] == B and q.shape[3] == D,
              f"q: [{B}, rows, heads, {D}] is required")
        R, H = q.shape[1], q.shape[2]
        _tensor(q, "q", self.dtype, (B, R, H, D), self.device)
        _need(R >= 1 and H >= K and H % K == 0, f"q: heads must be a multiple of the cache's {K}")
        _need(q.stride(3) == 1, "q: the last axis must be contiguous")
        _ints(kv_len, "kv_len", (B,), self.device)
        if rows is not None:
            _ints(rows, "rows", (B,), self.device)
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
                              A.addr(rows), R, H, int(bool(causal)), 1.0 / math.sqrt(D) if scale is None else scale)

    def attend(self, q, kv_len, *, k_new=None, v_new=None, rows=None, causal=True, scale: Optional[float] = None,
               out=None, lse=None):
        """Attention of the block's rows ``q [B, R, H, D]`` over the cache; ``k_new`` / ``v_new`` ``[B, R, K, D]`` are
        appended at ``kv_len``.  ``rows`` (int32 ``[B]``) are the rows in use.  Causal: row i sees slots 0 .. kv_len + i;
        else slots below kv_len.  Returns ``(out [B, R, H, D], lse [B, R, H])``; ``scale`` defaults to 1 / sqrt(D)."""
        r = self._rows(q, kv_len, rows, k_new, v_new, causal, scale)
        B, R, H, D = q.shape
        with torch.cuda.device(self.device):
            if out is None:
                out = torch.empty((B, R, H, D), dtype=self.dtype, device=self.device)
            else:
                _tensor(out, "out", self.dtype, (B, R, H, D), self.device)
                _need(out.is_contiguous(), "out: must be contiguous")
            if lse is None:
                lse = torch.empty((B, R, H), dtype=torch.float32, device=self.device)
            else:
                _tensor(lse, "lse", torch.float32, (B, R, H), self.device)
                _need(lse.is_contiguous(), "lse: must be contiguous")
            n = self._ws.get((R, H))
            if n is None:
                n = _check(A.lib().asr_spec_paged_attend_ws(self._ref, ctypes.byref(r)), "asr_spec_paged_attend_ws")
                self._ws[(R, H)] = n
            ws = torch.empty(n, dtype=torch.uint8, device=self.device)
            A.asr_spec_paged_attend(self._ref, r, out, lse, ws, n, torch.cuda.current_stream().cuda_stream)
        return out, lse

    def weigh(self, q, lse, kv_len, score, *, rows=None, causal=True, scale: Optional[float] = None, out=None, pos=None,
              first_pos=None):
        """Add the attention weight that the first ``rows`` rows gave each slot to ``score`` ``[B, K, slots]`` (fp32;
        None: zeros, then ``out`` is required).  Call it after the verification with the committed rows, and the
        ``kv_len`` and ``lse`` of the attention.  Writes ``out`` (default: ``score`` in place) and, with ``pos`` (int32,
        as score) and ``first_pos`` (int32 ``[B]``), the new slots' positions.  Returns ``out``."""
        r = self._rows(q, kv_len, rows, None, None, causal, scale)
        B, R, H = q.shape[:3]
        out = score if out is None else out
        _need(out is not None, "out: required without score")
        _need(out.dim() == 3, "score: [batch, kv_heads, slots] is required")
        shape = (B, self.kv_heads, out.shape[2])
        _tensor(out, "out", torch.float32, shape, self.device)
        _need(out.stride(2) == 1, "out: the last axis must be contiguous")
        for x, name, dt in ((score, "score", torch.float32), (pos, "pos", torch.int32)):
            if x is not None:
                _tensor(x, name, dt, shape, self.device)
                _need(x.stride() == out.stride(), f"{name}: out's strides are required")
        _need((pos is None) == (first_pos is None), "pos and first_pos go together")
        if first_pos is not None:
            _ints(first_pos, "first_pos", (B,), self.device)
        _tensor(lse, "lse", torch.float32, (B, R, H), self.device)
        _need(lse.stride(2) == 1, "lse: the last axis must be contiguous")
        s = A.AsrPagedScores(A.addr(score), A.addr(pos), out.stride(0), out.stride(1), shape[2], out.data_ptr(), None, 0, 0, 0,
                             A.addr(first_pos))
        with torch.cuda.device(self.device):
            A.asr_spec_paged_weigh(self._ref, r, s, lse, lse.stride(0), lse.stride(1), torch.cuda.current_stream().cuda_stream)
        return out

    def evict(self, lens, score, pos, seen, *, budget: int, recent: int = 0, first: int = 0, lens_out=None, score_out=None,
              pos_out=None):
        """Cut every head to its ``budget`` slots of highest accumulated weight; the ``recent`` newest positions
        (of ``seen`` ``[B]`` tokens) and the ``first`` oldest go last.  Freed slots below the budget take the kept ones
        past it.  ``score`` / ``pos`` ``[B, K, slots]`` and the pages' K/V move along: into ``score_out`` / ``pos_out``
        (default: in place) and in place.  Returns ``(lens_out, score_out, pos_out)``."""
        B, K = self.batch, self.kv_heads
        _ints(lens, "lens", (B,), self.device)
        _ints(seen, "seen", (B,), self.device)
        _need(isinstance(score, torch.Tensor) and score.dim() == 3, "score: [batch, kv_heads, slots] is required")
        _tensor(score, "score", torch.float32, (B, K, score.shape[2]), self.device)
        _tensor(pos, "pos", torch.int32, score.shape, self.device)
        score_out = score if score_out is None else score_out
        pos_out = pos if pos_out is None else pos_out
        _need(isinstance(score_out, torch.Tensor) and score_out.dim() == 3, "score_out: [batch, kv_heads, slots] is required")
        _tensor(score_out, "score_out", torch.float32, (B, K, score_out.shape[2]), self.device)
        _tensor(pos_out, "pos_out", torch.int32, score_out.shape, self.device)
        _need(score.stride() == pos.stride() and score.stride(2) == 1 and score_out.stride() == pos_out.stride() and
              score_out.stride(2) == 1, "score and pos: the same strides and a contiguous last axis are required")
        _need(budget >= 1 and recent >= 0 and first >= 0, "budget >= 1, recent >= 0 and first >= 0 are required")
        with torch.cuda.device(self.device):
            if lens_out is None:
                lens_out = torch.empty_like(lens)
            else:
                _ints(lens_out, "lens_out", (B,), self.device)
            s = A.AsrPagedScores(score.data_ptr(), pos.data_ptr(), score.stride(0), score.stride(1), score.shape[2],
                                 score_out.data_ptr(), pos_out.data_ptr(), score_out.stride(0), score_out.stride(1),
                                 score_out.shape[2], None)
            n = _check(A.lib().asr_spec_paged_evict_ws(self._ref, ctypes.byref(s), budget), "asr_spec_paged_evict_ws")
            ws = torch.empty(n, dtype=torch.uint8, device=self.device)
            A.asr_spec_paged_evict(self._ref, s, lens, seen, budget, recent, first, lens_out, ws, n,
                                   torch.cuda.current_stream().cuda_stream)
        return lens_out, score_out, pos_out


def accept_sampled(target, draft, lens, u, race, *, draft_logits=None, temperature: float = 1.0, status=None):
    """Accept drafted tokens against the target's probabilities from given random numbers.

    ``target [B, k + 1, V]`` and ``draft_logits [B, k, V]`` (None: greedy drafts) are logits of one type (float32,
    bfloat16, float16); ``draft [B, k]`` and ``lens [B]`` (-1 sits out; None: k each) are int32; ``u [B, k]`` uniform in
    [0, 1) and ``race [B, V]`` standard exponential, float32.  Returns ``(accepted [B], token [B], step [B], prob [B, k])``:
    the drafts accepted, the token drawn after them, the positions to commit and each draft's acceptance probability.
    ``status``: an int32 device tensor that collects ``asrspec.ST_*`` bits."""
    _need(isinstance(target, torch.Tensor) and target.is_cuda and target.dim() == 3 and target.dtype in _DTYPE,
          "target: [batch, k + 1, vocab] of float32, bfloat16 or float16 on a CUDA device is required")
    dev = target.device
    B, k, V = target.shape[0], target.shape[1] - 1, target.shape[2]
    _need(0 <= k <= 31 and B >= 1 and V >= 1, "target: 1 to 32 rows are required")
    _need(target.stride(2) == 1, "target: the last axis must be contiguous")
    _ints(draft, "draft", (B, k), dev)
    if lens is not None:
        _ints(lens, "lens", (B,), dev)
    _tensor(u, "u", torch.float32, (B, k), dev)
    _need(u.is_contiguous(), "u: must be contiguous")
    _tensor(race, "race", torch.float32, (B, V), dev)
    _need(race.stride(1) == 1, "race: the last axis must be contiguous")
    ds = (0, 0)
    if draft_logits is not None:
        _tensor(draft_logits, "draft_logits", target.dtype, (B, k, V), dev)
        _need(k == 0 or draft_logits.stride(2) == 1, "draft_logits: the last axis must be contiguous")
        ds = draft_logits.stride()[:2]
    if status is not None:
        _ints(status, "status", (1,), dev)
    _need(temperature > 0 and math.isfinite(temperature), "temperature: a positive number is required")
    with torch.cuda.device(dev):
        ints = torch.empty((3, B), dtype=torch.int32, device=dev)
        prob = torch.empty((B, k), dtype=torch.float32, device=dev)
        n = _check(A.lib().asr_spec_accept_sampled_ws(B, k), "asr_spec_accept_sampled_ws")
        ws = torch.empty(n, dtype=torch.uint8, device=dev)
        x = A.AsrSampledLogits(target.data_ptr(), target.stride(0), target.stride(1), A.addr(draft_logits) if k else None, *ds,
                               B, k, V, _DTYPE[target.dtype])
        accepted, token, step = ints.unbind(0)
        A.asr_spec_accept_sampled(x, draft, lens, u, race, race.stride(0), temperature, accepted, token, step, prob, status, ws,
                                  n, torch.cuda.current_stream().cuda_stream)
    return accepted, token, step, prob
