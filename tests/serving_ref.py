"""Plain 64-bit implementations of the operators over a paged cache, one
sequence and one head at a time, and the error bounds of the kernels' types."""
import math

import numpy as np
import torch

EPS_OUT = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}   # half the spacing just above 1


def slots(pages, table_row, n):
    """[n, K, D] float64 of a sequence's first n slots, page by page."""
    page = pages.shape[2]
    got = [pages[int(table_row[j])].transpose(0, 1)[:min(page, n - j * page)] for j in range(-(-n // page))]
    return torch.cat(got).double() if got else torch.zeros((0, pages.shape[1], pages.shape[3]), dtype=torch.float64,
                                                           device=pages.device)


def score_bound(q, k, scale):
    """Largest error of one score: D products accumulated in fp32, with truncation at every step allowed for."""
    D = q.shape[-1]
    return (D + 8) * 2.0 ** -22 * scale * (k.abs() @ q.abs())


def attend(q, k_pages, v_pages, table, kv_len, rows, k_new, v_new, causal, scale):
    """Returns out, lse, bound on out, bound on lse (float64) and writes the new rows into the pages given."""
    B, R, H, D = q.shape
    K = k_pages.shape[1]
    page = k_pages.shape[2]
    dt = q.dtype
    out = torch.zeros((B, R, H, D), dtype=torch.float64, device=q.device)
    lse = torch.full((B, R, H), -math.inf, dtype=torch.float64, device=q.device)
    ob, lb = torch.zeros_like(out), torch.zeros_like(lse)
    for b in range(B):
        n, r = int(kv_len[b]), int(rows[b])
        if k_new is not None:
            for i in range(r):
                at = n + i
                k_pages[int(table[b, at // page]), :, at % page] = k_new[b, i]
                v_pages[int(table[b, at // page]), :, at % page] = v_new[b, i]
        for i in range(r):
            end = n + i + 1 if causal else n
            if end == 0:
                continue
            k, v = slots(k_pages, table[b], end), slots(v_pages, table[b], end)
            for h in range(H):
                kk, vv, qq = k[:, h // (H // K)], v[:, h // (H // K)], q[b, i, h].double()
                x = scale * (kk @ qq)
                l = torch.logsumexp(x, 0)
                p = torch.exp(x - l)
                out[b, i, h] = p @ vv
                lse[b, i, h] = l
                ds = score_bound(qq, kk, scale).max()
                lb[b, i, h] = ds + 2.0 ** -20 * (1 + l.abs() + x.abs().max())
                # weights: the scores' error twice (numerator, sum), exp2 and its argument, the rounding of p
                # to 16 bits; sums of `end` fp32 terms; the output's own rounding
                rel = 2 * ds + 2.0 ** -20 * (1 + x.abs().max()) + (0.0 if dt == torch.float32 else EPS_OUT[dt]) \
                    + end * 2.0 ** -23
                ob[b, i, h] = rel * (p @ vv.abs()) + EPS_OUT[dt] * out[b, i, h].abs() * 1.01 + 1e-30
                if dt == torch.float16:
                    ob[b, i, h] += 2.0 ** -24   # subnormal weights and outputs
    return out, lse, ob, lb


def weigh(q, lse, k_pages, table, kv_len, rows, score, causal, scale):
    """New scores [B, K, slots] and their bounds; entries past the last slot keep NaN."""
    B, R, H, D = q.shape
    K = k_pages.shape[1]
    out = torch.full(score.shape, math.nan, dtype=torch.float64, device=q.device)
    bound = torch.zeros_like(out)
    for b in range(B):
        n, r = int(kv_len[b]), int(rows[b])
        end = n + r if causal else n
        k = slots(k_pages, table[b], end)
        out[b, :, :end] = 0
        out[b, :, :min(n, end)] = score[b, :, :min(n, end)].double()
        for i in range(r):
            e = n + i + 1 if causal else n
            for h in range(H):
                if not math.isfinite(float(lse[b, i, h])):
                    continue
                g = h // (H // K)
                x = scale * (k[:e, g] @ q[b, i, h].double())
                w = torch.exp(x - lse[b, i, h].double())
                out[b, g, :e] += w
                bound[b, g, :e] += w * (score_bound(q[b, i, h].double(), k[:e, g], scale) +
                                        2.0 ** -20 * (1 + x.abs() + lse[b, i, h].double().abs()))
        bound[b, :, :end] += (R * H // K + 2) * 2.0 ** -23 * out[b, :, :end].abs()
    return out, bound


def evict(lens, score, pos, seen, budget, recent, first):
    """Per (sequence, head): the kept slots' new order as a list of source slots."""
    B, K = score.shape[:2]
    plan = [[None] * K for _ in range(B)]
    for b in range(B):
        n = int(lens[b])
        for h in range(K):
            order = list(range(n))
            if n > budget:
                def rank(i):
                    s, p = float(score[b, h, i]), int(pos[b, h, i])
                    safe = p >= int(seen[b]) - recent or p < first
                    return (0 if safe else 1, 0.0 if safe else (math.inf if math.isnan(s) else -s), i)
                keep = set(sorted(range(n), key=lambda i: (rank(i)[0], 1 if not rank(i)[0] == 0 and
                                                          math.isnan(float(score[b, h, i])) else 0, rank(i)[1], i))[:budget])
                holes = [i for i in range(budget) if i not in keep]
                past = [i for i in range(budget, n) if i in keep]
                order = list(range(budget))
                for to, of in zip(holes, past):
                    order[to] = of
            plan[b][h] = order
    return plan


def softmax64(row, temperature):
    """Probabilities of one row: NaN and -inf masked, +inf the largest float; all masked: zeros."""
    x = np.asarray(row, dtype=np.float64).copy()
    x[np.isnan(x)] = -np.inf
    x = np.minimum(x, float(np.finfo(np.float32).max))
    if not np.isfinite(x.max()):
        return np.zeros_like(x)
    e = np.exp((x - x.max()) / temperature)
    return e / e.sum()


def accept(target, draft, lens, u, race, draft_logits, temperature):
    """accepted, token, step, prob and the smallest relative margin of any decision of each utterance."""
    B, k, V = target.shape[0], target.shape[1] - 1, target.shape[2]
    acc, tok, step, prob = np.zeros(B, int), np.full(B, -1), np.zeros(B, int), np.zeros((B, k))
    margin = np.full(B, np.inf)
    for b in range(B):
        if lens[b] < 0:
            continue
        p = [softmax64(target[b, i], temperature) for i in range(lens[b] + 1)]
        q = []
        for i in range(lens[b]):
            if draft_logits is None:
                q.append(np.eye(1, V, draft[b, i])[0])
            else:
                q.append(softmax64(draft_logits[b, i], temperature))
            px, qx = p[i][draft[b, i]], q[i][draft[b, i]]
            prob[b, i] = min(1.0, px / qx) if qx > 0 else float(px > 0)
        n = 0
        while n < lens[b]:
            px, qx = p[n][draft[b, n]], q[n][draft[b, n]]
            if px > 0:
                margin[b] = min(margin[b], abs(u[b, n] * qx - px) / px)
            if not u[b, n] * qx < px:
                break
            n += 1
        w = np.maximum(p[n] - q[n], 0) if n < lens[b] else p[n]
        if not w.max() > 0:
            w = p[n]
        acc[b] = n
        if w.max() > 0:
            x = w / race[b].astype(np.float64)
            tok[b], step[b] = int(x.argmax()), n + 1
            two = np.sort(x)[-2:]
            if V > 1 and two[-1] > 0:
                margin[b] = min(margin[b], (two[-1] - two[0]) / two[-1])
    return acc, tok, step, prob, margin
