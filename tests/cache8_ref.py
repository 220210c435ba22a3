"""Plain 64-bit implementations of the operators of an 8-bit paged cache, of the
pages of a pool and of the adjustment of logits, one sequence at a time, and the
error bounds of the attention."""
import math

import numpy as np
import torch

from serving_ref import EPS_OUT

GROUP = 16


def scale_for(amax):
    """The least 2^e >= 2^-126 with amax <= 448 * 2^e."""
    if not amax > 0:
        return 2.0 ** -126
    e = math.ceil(math.log2(amax / 448.0)) - 1
    while 448.0 * 2.0 ** e < amax:
        e += 1
    return 2.0 ** max(e, -126)


def append(pages, scales, table, lens, rows, new):
    """Codes and scales of the appended rows, group by group, in place; lens and rows are lists."""
    page = pages.shape[2]
    for b, (n, r) in enumerate(zip(lens, rows)):
        for g in range(n // GROUP, (n + r - 1) // GROUP + 1 if r else 0):
            pid, at = int(table[b, g * GROUP // page]), g * GROUP % page
            lo, hi = max(n, g * GROUP), min(n + r, (g + 1) * GROUP)
            for h in range(pages.shape[1]):
                x = new[b, lo - n:hi - n, h].double()
                ok = torch.isfinite(x)
                s = scale_for(float(x.abs()[ok].max()) if bool(ok.any()) else 0.0)
                x = torch.where(ok, x, math.nan)
                if lo > g * GROUP:
                    was = float(scales[pid, h, at // GROUP])
                    s = max(s, was)
                    x = torch.cat([pages[pid, h, at:at + lo - g * GROUP].double() * was, x])
                pages[pid, h, at:at + x.shape[0]] = (x / s).float().to(torch.float8_e4m3fn)
                scales[pid, h, at // GROUP] = s


def slots(pages, scales, table_row, n):
    """[n, K, D] float64 of a sequence's first n slots, and their scales [n, K]."""
    page = pages.shape[2]
    x, s = [], []
    for j in range(-(-n // page)):
        m, pid = min(page, n - j * page), int(table_row[j])
        g = scales[pid].double().repeat_interleave(GROUP, dim=1).T[:m]
        x.append(pages[pid].transpose(0, 1)[:m].double() * g[..., None])
        s.append(g)
    return torch.cat(x), torch.cat(s)


def attend(q, k, v, ks, vs, table, lens, rows, causal, scale):
    """out, lse and bounds on both (float64), of rows whose K/V are in the pages already."""
    B, R, H, D = q.shape
    G = H // k.shape[1]
    out = torch.zeros((B, R, H, D), dtype=torch.float64, device=q.device)
    lse = torch.full((B, R, H), -math.inf, dtype=torch.float64, device=q.device)
    ob, lb = torch.zeros_like(out), torch.zeros_like(lse)
    for b in range(B):
        n, r = lens[b], rows[b]
        end = n + (r if causal else 0)
        if r == 0 or end == 0:
            continue
        kk, _ = slots(k, ks, table[b], end)
        vv, vg = slots(v, vs, table[b], end)
        # slots that row i sees, [r, 1]
        seen = (torch.arange(r, device=q.device) + n + 1 if causal else torch.full((r,), n, device=q.device))[:, None]
        hidden = torch.arange(end, device=q.device)[None, :] >= seen
        for h in range(H):
            kh, vh, qh = kk[:, h // G], vv[:, h // G], q[b, :r, h].double()
            x = (scale * (qh @ kh.T)).masked_fill(hidden, -math.inf)
            l = torch.logsumexp(x, 1)
            p = torch.exp(x - l[:, None])
            # a hidden slot adds nothing, whatever it holds
            bad = ~torch.isfinite(vh)
            o = p @ vh.masked_fill(bad, 0.0)
            o = torch.where((~hidden).double() @ bad.double() > 0, math.nan, o)
            out[b, :r, h], lse[b, :r, h] = o, l
            # scores: fp32 sums; exp2 and its argument; statistics in fp32
            ds = (D + 8) * 2.0 ** -22 * scale * (qh.abs() @ kh.abs().T).masked_fill(hidden, 0.0).amax(dim=1)
            most = x.abs().masked_fill(hidden, 0.0).amax(dim=1)
            lb[b, :r, h] = ds + 2.0 ** -20 * (1 + l.abs() + most) + seen[:, 0] * 2.0 ** -23
            # weights: the scores' error twice (numerator, sum), their rounding to fp16 (half a step, 2^-11 of the weight; a
            # subnormal one is off by half of 2^-24, and the largest of a row is 2^10 or more: 2^-35 of the largest weight times
            # scale, times codes of 448 at most), sums of `seen` fp32 terms, the output's own rounding
            rel = 2 * ds + 2.0 ** -20 * (1 + most) + 2.0 ** -11 + seen[:, 0] * 2.0 ** -23
            low = seen[:, 0] * 2.0 ** -35 * 448 * (p * vg[:, h // G][None, :]).amax(dim=1)
            bound = rel[:, None] * (p @ vh.abs().masked_fill(bad, 0.0)) + low[:, None] + EPS_OUT[q.dtype] * o.abs() * 1.01 + 1e-30
            if q.dtype == torch.float16:
                bound += 2.0 ** -25   # a subnormal output
            ob[b, :r, h] = bound
    return out, lse, ob, lb


# ---------------------------------------------------------------------- pools (numpy, host)
def reserve(table, held, refs, lens, rows, page):
    """table, held, refs, counts and copies [(source, destination, slots)] after a call, on copies of the arrays."""
    table, held, now, was = table.copy(), held.copy(), refs.copy(), refs
    free = [int(i) for i in np.flatnonzero(refs == 0)]
    tails = {}
    for b, (n, r) in enumerate(zip(lens, rows)):
        if r > 0 and n // page < held[b]:
            tails.setdefault(int(table[b, n // page]), []).append(b)
    taken, copies = 0, []
    for b, (n, r) in enumerate(zip(lens, rows)):
        if r <= 0:
            continue
        for j in range(n // page, (n + r - 1) // page + 1):
            old = int(table[b, j]) if j < held[b] else -1
            if old >= 0:
                if was[old] <= 1 or (j == n // page and len(tails[old]) == was[old] and tails[old][0] == b):
                    continue
                now[old] -= 1
            if taken == len(free):
                return None
            new, taken = free[taken], taken + 1
            now[new] += 1
            if old >= 0 and j == n // page and n % page:
                copies.append((old, new, n % page))
            table[b, j] = new
        held[b] = max(held[b], (n + r - 1) // page + 1)
    return table, held, now, (taken, len(free) - taken), copies


def fork(table, held, refs, parent, keep, page):
    """table, held, refs; entries past the new held ones are as they were.  Changes of the counts alone: other holders stay."""
    out, n_out, now = table.copy(), held.copy(), refs.copy()
    for b in range(len(held)):
        p = b if parent is None else parent[b]
        n = 0 if p < 0 else int(held[p])
        if keep is not None:
            n = min(n, -(-keep[b] // page))
        for j in range(held[b]):
            now[table[b, j]] -= 1
        for j in range(n):
            out[b, j] = table[p, j]
            now[table[p, j]] += 1
        n_out[b] = n
    return out, n_out, now


def compact(table, held, refs):
    """table, refs, where, live and moves [(source, destination)]."""
    live = int((refs > 0).sum())
    dst, src = np.flatnonzero(refs[:live] <= 0), live + np.flatnonzero(refs[live:] > 0)
    where = np.where(refs > 0, np.arange(refs.size), -1).astype(np.int32)
    where[src] = dst
    now, out = np.zeros_like(refs), table.copy()
    for old, new in enumerate(where):
        if new >= 0:
            now[new] = refs[old]
    for b, h in enumerate(held):
        out[b, :h] = where[table[b, :h]]
    return out, now, where, live, list(zip(src.tolist(), dst.tolist()))


# ---------------------------------------------------------------------- logits (numpy, host)
def adjust(logits, history, seen, prompt, draft, lens, rep, freq, pres, bias, mask):
    """[B, R, V] float64 and an error bound of fp32 arithmetic; rows past lens are NaN in both."""
    B, R, V = logits.shape
    out, bound = np.full((B, R, V), np.nan), np.full((B, R, V), np.nan)
    for b in range(B):
        for i in range(lens[b] + 1):
            said = list(history[b, prompt[b]:seen[b]]) + list(draft[b, :i])
            every = [t for t in list(history[b, :prompt[b]]) + said if 0 <= t < V]
            said = [t for t in said if 0 <= t < V]
            count = np.bincount(np.array(said, dtype=np.int64), minlength=V).astype(np.float64)
            x = logits[b, i].astype(np.float64)
            at = np.unique(np.array(every, dtype=np.int64))
            x[at] = np.where(x[at] > 0, x[at] / rep[b], x[at] * rep[b])
            with np.errstate(invalid="ignore"):
                # four fp32 operations, each within half a step of the largest value that takes part
                size = np.abs(x) + np.abs(freq[b]) * count + np.abs(pres[b])
                x = x - freq[b] * count - pres[b] * (count > 0)
                if bias is not None:
                    row = (bias[b] if bias.ndim == 2 else bias).astype(np.float64)
                    size = size + np.abs(row)
                    x = x + row
            if mask is not None:
                bits = np.unpackbits(np.ascontiguousarray(mask[b, i]).view(np.uint8), bitorder="little")[:V]
                x[bits == 0] = -np.inf
            out[b, i], bound[b, i] = x, 5 * 2.0 ** -24 * size
    return out, bound
