"""The cases on which the operators of sampled decoding over a paged cache are measured.

Four operators: attention of a block of new rows over a paged K/V cache, appending the
block's K/V (``attend``); the attention weight that each cached slot received from the
committed rows (``weigh``); eviction of the least attended slots down to a budget
(``evict``); and acceptance of drafted tokens against the target's probabilities from
given random numbers (``accept``).  ``run`` is one call of one of them: with ``own`` through
the package, else in elementary torch operations in 32 bits.  ``exact`` is the operators'
definition in 64 bits.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

DTYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
BYTES = {"fp32": 4, "bf16": 2, "fp16": 2}


# ------------------------------------------------------------------------------- the cases
def _attend(name, dtype, batch, rows, heads, kv_heads, dim, page, lo, hi, causal=True):
    return dict(name=name, op="attend", dtype=dtype, batch=batch, rows=rows, heads=heads, kv_heads=kv_heads, dim=dim,
                page=page, lo=lo, hi=hi, causal=causal)


def _weigh(name, dtype, batch, rows, heads, kv_heads, dim, page, lo, hi):
    return dict(name=name, op="weigh", dtype=dtype, batch=batch, rows=rows, heads=heads, kv_heads=kv_heads, dim=dim,
                page=page, lo=lo, hi=hi)


def _evict(name, dtype, batch, kv_heads, dim, page, lo, hi, budget, recent, first):
    return dict(name=name, op="evict", dtype=dtype, batch=batch, kv_heads=kv_heads, dim=dim, page=page, lo=lo, hi=hi,
                budget=budget, recent=recent, first=first)


def _accept(name, dtype, batch, k, vocab, logits, temperature):
    return dict(name=name, op="accept", dtype=dtype, batch=batch, k=k, vocab=vocab, draft_logits=logits,
                temperature=temperature)


def listed():
    return [
        # one utterance, one new token, no drafts: the smallest step of the large decoder, where latency is all
        _attend("attend-token-b1", "bf16", 1, 1, 20, 20, 64, 64, 230, 230),
        # one utterance, 8 drafts and the pending token, after hours of transcript kept in the cache
        _attend("attend-block-b1-long", "bf16", 1, 9, 20, 20, 64, 64, 100001, 100001),
        # the batch-64 workload: 6 drafts, every utterance at its own length within the 448-token context
        _attend("attend-block-b64", "bf16", 64, 7, 20, 20, 64, 16, 4, 448),
        # the tiny fp32 decoder, 4 drafts, a batch of mixed lengths
        _attend("attend-block-fp32", "fp32", 32, 5, 6, 6, 64, 16, 0, 448),
        # cross-attention of a draft block over encoder frames kept in pages; an utterance without frames has empty rows
        _attend("attend-frames-b32", "bf16", 32, 9, 12, 12, 64, 32, 0, 1500, causal=False),
        # serving with grouped heads: one token each for many long sequences
        _attend("attend-grouped-long", "fp16", 48, 1, 32, 8, 128, 128, 1, 40000),
        # after a verification of the batch-64 workload: the committed rows' weights
        _weigh("weigh-block-b64", "bf16", 64, 7, 20, 20, 64, 16, 4, 448),
        # the same for single tokens of long sequences with grouped heads
        _weigh("weigh-grouped-long", "bf16", 8, 1, 32, 8, 128, 128, 20000, 40000),
        # the batch-64 workload held to 256 slots a head; utterances below the budget stay as they are
        _evict("evict-b64", "bf16", 64, 20, 64, 16, 200, 448, 256, 32, 4),
        # long sequences cut to a budget of 16384 slots a head
        _evict("evict-grouped-long", "fp16", 8, 8, 128, 128, 30001, 40000, 16384, 128, 4),
        # one utterance, 8 greedy drafts (no draft probabilities)
        _accept("accept-greedy-b1", "fp32", 1, 8, 51866, False, 1.0),
        # the batch-64 workload with sampled drafts and their logits
        _accept("accept-logits-b64", "fp32", 64, 6, 51866, True, 0.8),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49)))))))


def draw(rng):
    op = rng.choice(["attend", "attend", "weigh", "evict", "accept", "accept"])
    if op == "accept":
        dtype = rng.choice(["fp32", "fp32", "bf16", "fp16"])
        return dict(op=op, dtype=dtype, batch=_log(rng, 1, 64), k=_log(rng, 1, 16),
                    vocab=rng.choice([51865, 51866, _log(rng, 1000, 60000)]), draft_logits=rng.random() < 0.6,
                    temperature=rng.choice([0.3, 0.7, 1.0, 1.0, 1.3]))
    dtype = rng.choice(["bf16", "bf16", "fp16", "fp32"])
    dim = rng.choice([64, 64, 128])
    page = 16 * _log(rng, 1, 16)
    if dim == 128 or rng.random() < 0.3:
        kv_heads = _log(rng, 1, 16)
        heads = kv_heads * rng.choice([1, 2, 3, 4, 8])
    else:
        kv_heads = heads = _log(rng, 2, 24)
    batch = _log(rng, 1, 64)
    # a share of the largest listed case's bytes, spread over its logarithm
    slots = math.exp(rng.uniform(math.log(2e4), math.log(2.0e9))) / (2 * BYTES[dtype] * dim * kv_heads * batch)
    hi = int(max(17, min(120000, slots)))
    lo = rng.choice([0, hi // 3, hi])
    if op == "evict":
        lo = max(lo, 1)
        budget = max(8, int(rng.uniform(0.3, 0.95) * hi))
        return dict(op=op, dtype=dtype, batch=batch, kv_heads=kv_heads, dim=dim, page=page, lo=lo, hi=hi,
                    budget=budget, recent=rng.choice([0, 1, budget // 4]), first=rng.choice([0, 4]))
    rows = rng.choice([1, _log(rng, 1, 17)])
    case = dict(op=op, dtype=dtype, batch=batch, rows=rows, heads=heads, kv_heads=kv_heads, dim=dim, page=page, lo=lo,
                hi=hi)
    if op == "attend":
        case["causal"] = rng.random() < 0.75
    return case


# -------------------------------------------------------- sizes that follow from a case alone
def _lens(case):
    """Slots in use of each sequence, spread over [lo, hi] (both ends included from two sequences on)."""
    lo, hi, n = case["lo"], case["hi"], case["batch"]
    if n == 1:
        return [hi]
    at = [(i * 0.6180339887498949) % 1.0 for i in range(n)]
    at[0], at[-1] = 0.0, 1.0
    return [lo + int(round(x * (hi - lo))) for x in at]


def _rows(case):
    """Rows in use of each sequence: all of them in a batch of one, else from none to all."""
    n, r = case["batch"], case["rows"]
    if n == 1 or r == 1:
        return [r] * n
    return [r - (i * 7 % (r + 1) if i % 3 == 2 else 0) for i in range(n)]


def _drafts(case):
    """Drafts of each utterance: all k for most, fewer for some, none or sitting out for a few of a batch."""
    n, k = case["batch"], case["k"]
    return [k if i % 4 != 3 else (i * 5 % (k + 2)) - 1 for i in range(n)]


def work(case):
    if case["op"] == "accept":
        es, V = BYTES[case["dtype"]], case["vocab"]
        lens = _drafts(case)
        live = [x for x in lens if x >= 0]
        rows = sum(x + 1 for x in live) + (sum(live) if case["draft_logits"] else 0)
        return {"bytes": rows * V * es + len(live) * V * 4 + case["batch"] * (case["k"] * 12 + 20),
                "flops": 4 * rows * V + 6 * len(live) * V}
    es, D, K = BYTES[case["dtype"]], case["dim"], case["kv_heads"]
    lens = _lens(case)
    if case["op"] == "evict":
        moved = sum(case["budget"] * (n - case["budget"]) // n for n in lens if n > case["budget"]) * K   # any order of scores
        return {"bytes": 2 * 2 * moved * D * es + sum(lens) * K * 8 + sum(min(n, case["budget"]) for n in lens) * K * 8,
                "flops": 4 * sum(lens) * K}
    rows, H = _rows(case), case["heads"]
    if case["op"] == "attend":
        new = rows if case["causal"] else [0] * len(rows)
        b = sum(n * 2 * K * D * es for n, r in zip(lens, rows) if r) + sum(new) * 4 * K * D * es
        b += sum(rows) * H * (2 * D * es + 4)
        return {"bytes": b, "flops": 4 * D * H * sum(r * (n + m) for n, r, m in zip(lens, rows, new))}
    b = sum((n + r) * K * ((D * es if r else 0) + 8) for n, r in zip(lens, rows)) + sum(rows) * H * (D * es + 4)
    return {"bytes": b, "flops": 2 * D * H * sum(r * (n + r) for n, r in zip(lens, rows))}


# ------------------------------------------------------------------------------- the inputs
def _ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _pages(case, g, slots):
    """A pool in use: every sequence's pages scattered over it, a few pages free; stale values past each length."""
    B, page = case["batch"], case["page"]
    per = -(-max(max(slots), 1) // page)
    need = [-(-n // page) for n in slots]
    n_pages = sum(need) + 3
    order = torch.randperm(n_pages, generator=g, device="cuda").to(torch.int32).tolist()
    table, at = [], 0
    for n in need:
        table.append(order[at:at + n] + [order[-1]] * (per - n))
        at += n
    shape = (n_pages, case["kv_heads"], page, case["dim"])
    k = torch.empty(shape, dtype=DTYPES[case["dtype"]], device="cuda").normal_(generator=g)
    v = torch.empty(shape, dtype=DTYPES[case["dtype"]], device="cuda").normal_(generator=g)
    return k, v, _ints(table).reshape(B, per)


def _inputs(case, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    dt = DTYPES[case["dtype"]]
    if case["op"] == "accept":
        B, k, V = case["batch"], case["k"], case["vocab"]
        lens = _drafts(case)

        def draw_(scale):
            return torch.empty((B, k + 1, V), device="cuda").normal_(generator=g) * scale

        base = draw_(2.0)
        # a few likely tokens in each row, as a speech decoder's: the mass sits on them
        likely = torch.randint(0, V, (B, k + 1, 4), generator=g, device="cuda")
        base.scatter_add_(2, likely, 10.0 + 4.0 * torch.rand((B, k + 1, 4), generator=g, device="cuda"))
        target = base.clone()
        suppressed = torch.randint(0, V, (V // 64,), generator=g, device="cuda")
        target[:, :, suppressed] = -math.inf
        s = {"target": target.to(dt), "draft_logits": None}
        noisy = base + draw_(0.5)
        if case["draft_logits"]:
            s["draft_logits"] = noisy[:, :k].contiguous().to(dt)
            e = torch.empty((B, k, V), device="cuda").exponential_(generator=g).clamp_(min=1e-30)
            noisy = s["draft_logits"].float() / case["temperature"] - e.log()
        s["draft"] = noisy[:, :k].argmax(dim=2).to(torch.int32)
        s["lens"] = _ints(lens)
        s["u"] = torch.rand((B, k), generator=g, device="cuda")
        s["race"] = torch.empty((B, V), device="cuda").exponential_(generator=g).clamp_(min=1e-30)
        return s
    lens = _lens(case)
    if case["op"] == "evict":
        k, v, table = _pages(case, g, lens)
        B, K = case["batch"], case["kv_heads"]
        cap = max(lens)
        # accumulated weights: heavy-tailed, with equal values among the rarely attended slots
        score = torch.empty((B, K, cap), device="cuda").log_normal_(mean=-2.0, std=2.0, generator=g)
        score = torch.where(score < 0.05, torch.round(score * 64) / 64, score)
        n = max(lens) + 500    # tokens seen: earlier evictions left gaps and an order of their own
        pos = torch.rand((B, K, n), generator=g, device="cuda").argsort(dim=2)[:, :, :cap].to(torch.int32)
        return {"k": k, "v": v, "table": table, "lens": _ints(lens), "score": score, "pos": pos.contiguous(),
                "seen": _ints([n] * B), "score_out": torch.zeros_like(score), "pos_out": torch.zeros_like(pos)}
    rows = _rows(case)
    causal = case.get("causal", True)
    B, R, H, K, D = case["batch"], case["rows"], case["heads"], case["kv_heads"], case["dim"]
    slots = [n + (R if causal else 0) for n in lens]
    k, v, table = _pages(case, g, slots)
    # one projection's output holds the rows' queries, keys and values side by side
    qkv = torch.empty((B, R, (H + 2 * K) * D), dtype=dt, device="cuda").normal_(generator=g)
    q = qkv[:, :, :H * D].unflatten(2, (H, D))
    q *= 1.5
    s = {"k": k, "v": v, "table": table, "lens": _ints(lens), "rows": _ints(rows), "q": q, "k_new": None,
         "v_new": None}
    if case["op"] == "attend" and causal:
        s["k_new"] = qkv[:, :, H * D:(H + K) * D].unflatten(2, (K, D))
        s["v_new"] = qkv[:, :, (H + K) * D:].unflatten(2, (K, D))
    if case["op"] == "weigh":
        cap = table.shape[1] * case["page"]
        s["lse"] = _row_lse(case, s)
        s["score"] = torch.empty((B, K, cap), device="cuda").exponential_(generator=g)
        s["score_out"] = torch.zeros_like(s["score"])
        s["pos"] = torch.randint(0, 1 << 20, (B, K, cap), generator=g, device="cuda", dtype=torch.int32)
        s["first_pos"] = _ints([3 * n + 1 for n in lens])
    return s


def _row_lse(case, s):
    """The rows' log-sum-exp, as the attention that came before left it (fp32)."""
    B, R, H, K = case["batch"], case["rows"], case["heads"], case["kv_heads"]
    out = torch.full((B, R, H), -math.inf, device="cuda")
    for b, (n, r) in enumerate(zip(_lens(case), _rows(case))):
        if r:
            k = _gather(s["k"], s["table"][b:b + 1], n + r)[0].float()
            out[b, :r] = torch.logsumexp(_scores(s["q"][b, :r].float(), k, n, True), dim=2).permute(1, 0)
    return out


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = case
    if own:
        from paper_2608_12703_gb300 import serving
        if case["op"] == "accept":
            s["accept"] = serving.accept_sampled
        else:
            s["cache"] = serving.PagedCache(s["k"], s["v"], s["table"])
    return s


# ------------------------------------------------------------------------- the plain forms
def _gather(pages, table, n):
    """[B, K, n, D] of the sequences' first n slots."""
    page = pages.shape[2]
    x = pages[table[:, :-(-n // page)].long()]                  # [B, p, K, page, D]
    return x.transpose(1, 2).flatten(2, 3)[:, :, :n]


def _scores(q, k, n, causal):
    """[H, r, keys] scaled scores of one sequence's rows q [r, H, D] over k [K, keys, D]."""
    r, H, D = q.shape
    K = k.shape[0]
    x = q.permute(1, 0, 2).reshape(K, (H // K) * r, D) @ k.transpose(1, 2) * (1.0 / math.sqrt(D))
    x = x.reshape(H, r, -1)
    if causal:
        slot = torch.arange(x.shape[2], device=x.device)
        row = torch.arange(r, device=x.device)
        x = x.masked_fill(slot[None, :] > n + row[:, None], -math.inf)
    return x


def _put(pages, table, new, lens, rows):
    """Write the rows' K or V behind each sequence's committed slots."""
    B, R = new.shape[:2]
    i = torch.arange(R, device="cuda")[None, :]
    slot = lens[:, None].long() + i
    page = table.long().gather(1, (slot // pages.shape[2]).clamp(max=table.shape[1] - 1))
    use = i < rows[:, None]
    pages[page[use], :, (slot % pages.shape[2])[use]] = new[use]


def _softmax_out(x, v):
    """Weighted values and log-sum-exp of masked scores x [..., keys]; an empty row gives zeros and -inf."""
    m = x.amax(dim=-1, keepdim=True)
    e = torch.exp(x - torch.where(torch.isinf(m), torch.zeros_like(m), m))
    l = e.sum(dim=-1, keepdim=True)
    o = (e @ v) / torch.where(l > 0, l, torch.ones_like(l))
    return o, (m + torch.log(l)).squeeze(-1)


def _attend_plain(case, s):
    B, R, H, K, D = case["batch"], case["rows"], case["heads"], case["kv_heads"], case["dim"]
    causal, G = case["causal"], case["heads"] // case["kv_heads"]
    if causal:
        _put(s["k"], s["table"], s["k_new"], s["lens"], s["rows"])
        _put(s["v"], s["table"], s["v_new"], s["lens"], s["rows"])
    out = torch.empty((B, R, H, D), dtype=s["q"].dtype, device="cuda")
    lse = torch.empty((B, R, H), device="cuda")
    most = s["table"].shape[1] * case["page"]
    step = max(1, int(3e8 // (K * D * most)))
    for b in range(0, B, step):
        t, n = s["table"][b:b + step], s["lens"][b:b + step, None, None, None]
        r = s["rows"][b:b + step, None, None, None]
        k, v = _gather(s["k"], t, most), _gather(s["v"], t, most)
        q = s["q"][b:b + step].float().permute(0, 2, 1, 3).reshape(-1, K, G * R, D)
        x = (q @ k.float().transpose(2, 3) * (1.0 / math.sqrt(D))).reshape(-1, K, G, R, most).flatten(1, 2)
        slot = torch.arange(most, device="cuda")[None, None, None, :]
        row = torch.arange(R, device="cuda")[None, None, :, None]
        x = x.masked_fill((slot >= n + (row + 1 if causal else 0)) | (row >= r), -math.inf)
        v = torch.where(torch.arange(most, device="cuda")[None, None, :, None] < n + (r if causal else 0), v.float(), 0.0)
        o, l = _softmax_out(x.reshape(-1, K, G * R, most), v)
        out[b:b + step] = o.reshape(-1, H, R, D).permute(0, 2, 1, 3).to(out.dtype)
        lse[b:b + step] = l.reshape(-1, H, R).permute(0, 2, 1)
    return out, lse, s["k"], s["v"]


def _weigh_plain(case, s):
    B, R, H, K, D = case["batch"], case["rows"], case["heads"], case["kv_heads"], case["dim"]
    G = H // K
    cap = s["score"].shape[2]
    score, pos = s["score_out"], s["pos"]
    slot = torch.arange(cap, device="cuda")
    row = torch.arange(R, device="cuda")
    step = max(1, int(3e8 // (K * D * cap)))
    for b in range(0, B, step):
        n, r = s["lens"][b:b + step, None, None], s["rows"][b:b + step, None, None]
        k = _gather(s["k"], s["table"][b:b + step], cap).float()
        q = s["q"][b:b + step].float().permute(0, 2, 1, 3).reshape(-1, K, G * R, D)
        x = (q @ k.transpose(2, 3) * (1.0 / math.sqrt(D))).reshape(-1, H, R, cap)
        w = torch.exp(x - s["lse"][b:b + step].permute(0, 2, 1)[..., None])
        see = (slot <= n[..., None] + row[:, None]) & (row[:, None] < r[..., None])
        w = torch.where(see, w, 0.0).reshape(-1, K, G * R, cap).sum(dim=2)
        old = torch.where(slot < n, s["score"][b:b + step], 0.0)
        score[b:b + step] = torch.where(slot < n + r, old + w, score[b:b + step])
        fresh = (slot >= n) & (slot < n + r)
        at = s["first_pos"][b:b + step, None, None] + (slot - n)
        pos[b:b + step] = torch.where(fresh, at.to(torch.int32), pos[b:b + step])
    return score, pos


def _evict_plain(case, s):
    budget, page = case["budget"], case["page"]
    B, K, cap = s["score"].shape
    slot = torch.arange(cap, device="cuda")
    live = slot < s["lens"][:, None, None]
    kept = (s["pos"] >= (s["seen"] - case["recent"])[:, None, None]) | (s["pos"] < case["first"])
    key = torch.where(kept, torch.full_like(s["score"], math.inf), s["score"])
    key = torch.where(live, key, torch.full_like(key, -math.inf))
    order = torch.sort(key, dim=2, descending=True, stable=True).indices      # equal keys: the lowest slot first
    keep = torch.zeros((B, K, cap), dtype=torch.bool, device="cuda")
    keep.scatter_(2, order[:, :, :budget], True)
    keep &= live
    # the j-th freed slot below the budget takes the j-th kept slot at or past it
    below = slot < budget
    hole, src = live & below & ~keep, keep & ~below
    hb, hh, hs = torch.nonzero(hole, as_tuple=True)
    sb, sh, ss = torch.nonzero(src, as_tuple=True)
    many = s["lens"][hb] > budget
    hb, hh, hs = hb[many], hh[many], hs[many]
    to = s["table"][hb, hs // page].long()
    of = s["table"][sb, ss // page].long()
    for p in (s["k"], s["v"]):
        p[to, hh, hs % page] = p[of, sh, ss % page]
    lens = torch.minimum(s["lens"], torch.full_like(s["lens"], budget))
    held = slot < lens[:, None, None]
    for name in ("score", "pos"):
        x = s[name].clone()
        x[hb, hh, hs] = x[sb, sh, ss]
        s[name + "_out"] = torch.where(held, x, s[name + "_out"])
    return lens, s["score_out"], s["pos_out"], s["k"], s["v"]


def _probs(logits, temperature):
    m = logits.amax(dim=-1, keepdim=True)
    e = torch.exp((logits - torch.where(torch.isinf(m), torch.zeros_like(m), m)) / temperature)
    l = e.sum(dim=-1, keepdim=True)
    return e / torch.where(l > 0, l, torch.ones_like(l))


def _first_max(x):
    """The largest value of each row and its lowest index."""
    m = x.amax(dim=-1)
    i = torch.arange(x.shape[-1], device=x.device)
    return m, torch.where(x == m[..., None], i, x.shape[-1]).amin(dim=-1)


def _accept_rule(p, q, draft, lens, u, race):
    """p [B, k+1, V], q [B, k, V] or None (drafts that were certain)."""
    B, k, V = p.shape[0], p.shape[1] - 1, p.shape[2]
    x = draft.long()[..., None]
    px = p[:, :k].gather(2, x).squeeze(2)
    qx = torch.ones_like(px) if q is None else q.gather(2, x).squeeze(2)
    drafted = torch.arange(k, device=p.device)[None, :] < lens[:, None]
    take = (u.to(px.dtype) * qx < px) & drafted
    n = torch.cumprod(take.long(), dim=1).sum(dim=1)
    prob = torch.where(px >= qx, (px > 0).to(px.dtype), px / torch.where(qx > 0, qx, torch.ones_like(qx)))
    prob = torch.where(drafted, prob, torch.zeros_like(prob))
    rows = torch.arange(B, device=p.device)
    pn = p[rows, n]
    at = n.clamp(max=max(k - 1, 0))
    if q is None:
        minus = torch.zeros_like(pn).scatter_(1, x[rows, at], math.inf)
    else:
        minus = q[rows, at]
    rest = torch.where((n < lens)[:, None], (pn - minus).clamp(min=0.0), pn)
    best, token = _first_max(rest / race.to(rest.dtype))
    best_p, token_p = _first_max(pn / race.to(rest.dtype))
    token = torch.where(best > 0, token, torch.where(best_p > 0, token_p, torch.full_like(token, -1)))
    out = lens < 0
    n = torch.where(out, torch.zeros_like(n), n)
    token = torch.where(out, torch.full_like(token, -1), token)
    step = torch.where(token < 0, torch.zeros_like(n), n + 1)
    return n.to(torch.int32), token.to(torch.int32), step.to(torch.int32), prob


def _accept_plain(case, s):
    t = case["temperature"]
    p = _probs(s["target"].float(), t)
    q = None if s["draft_logits"] is None else _probs(s["draft_logits"].float(), t)
    return _accept_rule(p, q, s["draft"], s["lens"], s["u"], s["race"])


def run(s):
    case = s["case"]
    op = case["op"]
    if not own:
        return {"attend": _attend_plain, "weigh": _weigh_plain, "evict": _evict_plain, "accept": _accept_plain}[op](case, s)
    if op == "accept":
        return s["accept"](s["target"], s["draft"], s["lens"], s["u"], s["race"], draft_logits=s["draft_logits"],
                           temperature=case["temperature"])
    cache = s["cache"]
    if op == "attend":
        out, lse = cache.attend(s["q"], s["lens"], k_new=s["k_new"], v_new=s["v_new"], rows=s["rows"],
                                causal=case["causal"])
        return out, lse, s["k"], s["v"]
    if op == "weigh":
        score = cache.weigh(s["q"], s["lse"], s["lens"], s["score"], rows=s["rows"], out=s["score_out"], pos=s["pos"],
                            first_pos=s["first_pos"])
        return score, s["pos"]
    lens, score, pos = cache.evict(s["lens"], s["score"], s["pos"], s["seen"], budget=case["budget"],
                                   recent=case["recent"], first=case["first"], score_out=s["score_out"],
                                   pos_out=s["pos_out"])
    return lens, score, pos, s["k"], s["v"]


# --------------------------------------------------------- the definition in 64 bits
def exact(case, seed):
    s = _inputs(case, seed)
    op = case["op"]
    if op == "accept":
        return _accept_exact(case, s)
    if work(case)["flops"] > 3e11 or s["k"].numel() > 3e9:
        return None
    if op == "evict":
        return _evict_exact(case, s)
    B, R, H, K, D = case["batch"], case["rows"], case["heads"], case["kv_heads"], case["dim"]
    G, page, causal = H // K, case["page"], case.get("causal", True)
    lens, rows = _lens(case), _rows(case)
    table = s["table"].cpu().tolist()

    def walk(pages, b, n):
        """The first n slots of sequence b, page by page: [n, K, D]."""
        got = [pages[table[b][j]].transpose(0, 1)[:min(page, n - j * page)] for j in range(-(-n // page))]
        return torch.cat(got).double() if got else torch.zeros((0, K, D), dtype=torch.float64, device="cuda")

    if op == "attend":
        out = torch.zeros((B, R, H, D), dtype=torch.float64, device="cuda")
        lse = torch.full((B, R, H), -math.inf, dtype=torch.float64, device="cuda")
        for b in range(B):
            if causal:
                for i in range(rows[b]):
                    at = lens[b] + i
                    s["k"][table[b][at // page], :, at % page] = s["k_new"][b, i]
                    s["v"][table[b][at // page], :, at % page] = s["v_new"][b, i]
            n = lens[b] + (rows[b] if causal else 0)
            if not rows[b] or not n:
                continue
            k, v = walk(s["k"], b, n), walk(s["v"], b, n)
            for h in range(H):
                for i in range(rows[b]):
                    end = lens[b] + i + 1 if causal else n
                    x = (k[:end, h // G] @ s["q"][b, i, h].double()) / math.sqrt(D)
                    lse[b, i, h] = torch.logsumexp(x, 0)
                    out[b, i, h] = torch.exp(x - lse[b, i, h]) @ v[:end, h // G]
        return out, lse, s["k"], s["v"]
    score = s["score_out"].double()
    pos = s["pos"].clone()
    for b in range(B):
        n, r = lens[b], rows[b]
        k = walk(s["k"], b, n + r)
        new = torch.zeros((K, n + r), dtype=torch.float64, device="cuda")
        new[:, :n] = s["score"][b, :, :n].double()
        for i in range(r):
            for h in range(H):
                x = (k[:n + i + 1, h // G] @ s["q"][b, i, h].double()) / math.sqrt(D)
                new[h // G, :n + i + 1] += torch.exp(x - s["lse"][b, i, h].double())
            pos[b, :, n + i] = int(s["first_pos"][b]) + i
        score[b, :, :n + r] = new
    return score, pos


def _evict_exact(case, s):
    """By slots, one head at a time, on the host."""
    lens, page = _lens(case), case["page"]
    score, pos = s["score"].cpu().numpy(), s["pos"].cpu().numpy()
    so, po = s["score_out"].cpu().numpy().astype(np.float64), s["pos_out"].cpu().numpy()
    table, seen = s["table"].cpu().numpy(), s["seen"].cpu().numpy()
    budget = case["budget"]
    for b in range(case["batch"]):
        n = lens[b]
        for h in range(case["kv_heads"]):
            sc, ps = score[b, h, :n].copy(), pos[b, h, :n].copy()
            if n > budget:
                safe = (ps >= seen[b] - case["recent"]) | (ps < case["first"])
                rank = np.lexsort((np.arange(n), -sc.astype(np.float64), ~safe))
                keep = np.sort(rank[:budget])
                src = keep[keep >= budget]
                hole = np.setdiff1d(np.arange(budget), keep)
                sc[hole], ps[hole] = sc[src], ps[src]
                tp, fp = torch.from_numpy(table[b, hole // page]).long().cuda(), torch.from_numpy(table[b, src // page]).long().cuda()
                to, of = torch.from_numpy(hole % page).cuda(), torch.from_numpy(src % page).cuda()
                for p in (s["k"], s["v"]):
                    p[tp, h, to] = p[fp, h, of]
            m = min(n, budget)
            so[b, h, :m], po[b, h, :m] = sc[:m], ps[:m]
    cut = torch.tensor([min(n, budget) for n in lens], dtype=torch.int32)
    return cut, torch.from_numpy(so), torch.from_numpy(po), s["k"], s["v"]


def _accept_exact(case, s):
    """One utterance and one draft at a time."""
    B, k, t = case["batch"], case["k"], case["temperature"]
    lens = _drafts(case)
    draft, u = s["draft"].cpu().tolist(), s["u"].cpu().double().tolist()
    acc, tok, step = [0] * B, [-1] * B, [0] * B
    prob = torch.zeros((B, k), dtype=torch.float64)

    def softmax(row):
        row = row.double() / t
        e = torch.exp(row - row.max())
        return e / e.sum()

    for b in range(B):
        if lens[b] < 0:
            continue
        n, rest, stopped = 0, None, False
        for i in range(lens[b]):
            p, x = softmax(s["target"][b, i]), draft[b][i]
            if s["draft_logits"] is None:
                q = torch.zeros_like(p)
                q[x] = 1.0
            else:
                q = softmax(s["draft_logits"][b, i])
            px, qx = float(p[x]), float(q[x])
            prob[b, i] = min(1.0, px / qx) if qx > 0 else float(px > 0)
            if not stopped:
                if u[b][i] * qx < px:
                    n += 1
                else:
                    stopped, rest = True, (p - q).clamp(min=0.0)
        if not stopped:
            rest = softmax(s["target"][b, n])
        elif not float(rest.max()) > 0:
            rest = softmax(s["target"][b, n])
        tok[b] = int((rest / s["race"][b].double()).argmax())
        acc[b], step[b] = n, n + 1
    i32 = lambda x: torch.tensor(x, dtype=torch.int32)
    return i32(acc), i32(tok), i32(step), prob
