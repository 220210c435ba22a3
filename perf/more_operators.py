"""The cases on which the operators of an 8-bit paged cache, of its pages and of the logits are measured.

Five operators: attention of a block of new rows over a paged K/V cache held in 8 bits with a scale
for each group of 16 slots and head, quantising and appending the block's K/V (``attend8``); private
pages for the slots that a call is about to write, shared ones copied (``reserve``); sequences that go
on from other sequences' pages, or give theirs back (``fork``); live pages moved to the front of the
pool (``compact``); and penalties for repeated tokens, biases and grammar masks on the logits of a
block (``adjust``).  ``run`` is one call of one of them: with ``own`` through the package, else in
elementary torch operations in 32 bits.  ``exact`` is the operators' definition in 64 bits.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

DTYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16, "fp8": torch.float8_e4m3fn}
BYTES = {"fp32": 4, "bf16": 2, "fp16": 2, "fp8": 1}
GROUP = 16       # slots of a sequence that share a scale


# ------------------------------------------------------------------------------- the cases
def _attend8(name, dtype, batch, rows, heads, kv_heads, dim, page, lo, hi, causal=True):
    return dict(name=name, op="attend8", dtype=dtype, batch=batch, rows=rows, heads=heads, kv_heads=kv_heads, dim=dim,
                page=page, lo=lo, hi=hi, causal=causal)


def _pool(name, op, dtype, prompts, samples, layers, kv_heads, dim, page, lo, hi, **more):
    return dict(name=name, op=op, dtype=dtype, prompts=prompts, samples=samples, layers=layers, kv_heads=kv_heads,
                dim=dim, page=page, lo=lo, hi=hi, **more)


def _adjust(name, dtype, batch, k, vocab, history, bias, mask):
    return dict(name=name, op="adjust", dtype=dtype, batch=batch, k=k, vocab=vocab, history=history, bias=bias, mask=mask)


def listed():
    return [
        # one utterance, one new token of the large decoder: the smallest step, where latency is all
        _attend8("attend8-token-b1", "bf16", 1, 1, 20, 20, 64, 64, 230, 230),
        # the batch-64 workload: 6 drafts, every utterance at its own length within the 448-token context
        _attend8("attend8-block-b64", "bf16", 64, 7, 20, 20, 64, 16, 4, 448),
        # prompts: long transcripts of other sessions taken into the cache, some behind what is there already
        _attend8("attend8-prompt-b4", "bf16", 4, 2048, 20, 20, 64, 64, 0, 1000),
        # serving with grouped heads: one token each for many sequences, twice as long as 16 bits would hold
        _attend8("attend8-grouped-long", "fp16", 48, 1, 32, 8, 128, 128, 1, 80000),
        # eight samples of one utterance right after the fork: all but one take a copy of the last page; tiny fp32 decoder
        _pool("reserve-samples-b8", "reserve", "fp32", 1, 8, 4, 6, 64, 16, 200, 200, rows=5),
        # 64 utterances with 4 samples each, half of the small decoder's layers, after the fork that follows the prompt
        _pool("reserve-forked-b256", "reserve", "bf16", 64, 4, 6, 12, 64, 64, 4, 448, rows=9),
        # beams of 8 utterances change places after a step
        _pool("fork-beams-b40", "fork", "bf16", 8, 5, 1, 6, 64, 16, 4, 448, keep=False),
        # 1024 long sessions: some end, some go on from others, all give back the pages behind rejected drafts
        _pool("fork-sessions-b1024", "fork", "bf16", 256, 4, 1, 1, 64, 16, 1000, 40000, keep=True),
        # a small pool after some sessions ended: the tiny fp32 decoder
        _pool("compact-b16", "compact", "fp32", 16, 1, 4, 6, 64, 16, 4, 448, live=0.6),
        # the 8-bit pool of the large decoder, two thirds in use
        _pool("compact-8bit-b64", "compact", "fp8", 32, 2, 32, 20, 64, 64, 4, 448, live=0.66),
        # one utterance, 8 drafts, within a grammar
        _adjust("adjust-grammar-b1", "fp32", 1, 8, 51866, 200, False, True),
        # the batch-64 workload with suppressed tokens, penalties and a grammar
        _adjust("adjust-all-b64", "fp32", 64, 6, 51866, 448, True, True),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49)))))))


def draw(rng):
    op = rng.choice(["attend8", "attend8", "attend8", "reserve", "fork", "compact", "adjust", "adjust"])
    if op == "adjust":
        return dict(op=op, dtype=rng.choice(["fp32", "fp32", "bf16", "fp16"]), batch=_log(rng, 1, 64), k=_log(rng, 1, 16) - 1,
                    vocab=rng.choice([51865, 51866, _log(rng, 1000, 60000)]), history=_log(rng, 1, 4000),
                    bias=rng.random() < 0.5, mask=rng.random() < 0.6)
    dim = rng.choice([64, 64, 128])
    page = 16 * _log(rng, 1, 16)
    if op == "attend8":
        if dim == 128 or rng.random() < 0.3:
            kv_heads = _log(rng, 1, 16)
            heads = kv_heads * rng.choice([1, 2, 3, 4, 8])
        else:
            kv_heads = heads = _log(rng, 2, 24)
        batch = _log(rng, 1, 64)
        # a share of the largest listed case's bytes, spread over its logarithm
        slots = math.exp(rng.uniform(math.log(2e4), math.log(2.0e9))) / (2 * dim * kv_heads * batch)
        hi = int(max(17, min(200000, slots)))
        rows = rng.choice([1, _log(rng, 1, 17), _log(rng, 1, 17), _log(rng, 18, 2000)])
        # products of prompts are held to the listed prompts'
        rows = max(1, min(rows, int(2.0e10 / (dim * heads * batch * (hi + rows)))))
        return dict(op=op, dtype=rng.choice(["bf16", "bf16", "fp16"]), batch=batch, rows=rows, heads=heads,
                    kv_heads=kv_heads, dim=dim, page=page, lo=rng.choice([0, hi // 3, hi]), hi=hi,
                    causal=rng.random() < 0.75)
    dtype = rng.choice(["fp8", "bf16", "fp16", "fp32"])
    prompts, samples, kv_heads = _log(rng, 1, 64), _log(rng, 1, 8), _log(rng, 1, 24)
    if op == "fork":
        hi = _log(rng, 17, 20000)
        return dict(op=op, dtype="bf16", prompts=prompts, samples=samples, layers=1, kv_heads=1, dim=64,
                    page=page, lo=rng.choice([1, hi // 3, hi]), hi=hi, keep=rng.random() < 0.5)
    # a share of the largest listed pool
    total = math.exp(rng.uniform(math.log(3e6), math.log(2.5e9)))
    layers = _log(rng, 1, 32)
    per_page = 2 * layers * kv_heads * page * dim * BYTES[dtype]
    hi = int(max(17, min(4000, total / per_page / prompts / (3 if samples > 1 and op == "reserve" else 1) * page)))
    case = dict(op=op, dtype=dtype, prompts=prompts, samples=samples, layers=layers, kv_heads=kv_heads, dim=dim,
                page=page, lo=max(1, rng.choice([1, hi // 3, hi])), hi=hi)
    if op == "reserve":
        case["rows"] = _log(rng, 1, 17)
    else:
        case["live"] = rng.uniform(0.2, 0.95)
    while _pool_pages(case) * per_page > 4e9 and case["layers"] > 1:
        case["layers"] -= max(1, case["layers"] // 4)
        per_page = 2 * case["layers"] * kv_heads * page * dim * BYTES[dtype]
    while _pool_pages(case) * per_page > 4e9 and case["prompts"] > 1:
        case["prompts"] -= max(1, case["prompts"] // 4)
    return case


# -------------------------------------------------------- sizes that follow from a case alone
def _spread(lo, hi, n):
    """n lengths over [lo, hi], both ends included from two on."""
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


def _history(case):
    """(tokens seen, those of them that belong to the prompt) of each utterance."""
    n = _spread(min(4, case["history"]), case["history"], case["batch"])
    return n, [min(x, 4 + (i % 5) * 3) for i, x in enumerate(n)]


def _ceil(a, b):
    return -(-a // b)


def _pool_lens(case):
    """Slots of each sequence: the samples of a prompt are at the same length (reserve), or up to 40 tokens apart."""
    lens = [n for n in _spread(case["lo"], case["hi"], case["prompts"]) for _ in range(case["samples"])]
    if case["op"] == "reserve":
        return lens
    return [n + (i % case["samples"]) * 7 % 41 for i, n in enumerate(lens)]


def _pool_shape(case):
    """Pages of each sequence, those of them at the front that a prompt's samples share, and pages of a table row."""
    page, lens = case["page"], _pool_lens(case)
    held = [_ceil(n, page) for n in lens]
    first = [lens[i - i % case["samples"]] for i in range(len(lens))]
    shared = [h if case["op"] == "reserve" else min(h, n // page) for h, n in zip(held, first)]
    return held, shared, max(held) + _ceil(case.get("rows", 0), page) + 1


def _pool_live(case):
    """Pages in use."""
    held, shared, _ = _pool_shape(case)
    return sum(h if i % case["samples"] == 0 else h - s for i, (h, s) in enumerate(zip(held, shared)))


def _pool_pages(case):
    live = _pool_live(case)
    if case["op"] == "compact":
        return max(live + 1, int(live / case["live"]))
    if case["op"] == "reserve":
        return live + len(_pool_lens(case)) * (_ceil(case["rows"], case["page"]) + 1) + 3
    return live + 3


def _copied(case):
    """Slots that a call of reserve copies: each prompt's last page for all samples but one."""
    lens = _pool_lens(case)
    return sum(lens[i] % case["page"] for i in range(len(lens)) if i % case["samples"])


def _row_bytes(case):
    """Bytes of one slot's K and V in all layers, scales included."""
    return 2 * case["layers"] * case["kv_heads"] * (case["dim"] * BYTES[case["dtype"]] + (0.25 if case["dtype"] == "fp8" else 0))


def work(case):
    op = case["op"]
    if op == "adjust":
        es, V = BYTES[case["dtype"]], case["vocab"]
        rows = sum(n + 1 for n in _drafts(case))
        n = sum(_history(case)[0])
        return {"bytes": rows * V * es * 2 + (V * 4 if case["bias"] else 0) + (rows * V // 8 if case["mask"] else 0) + n * 4,
                "flops": 4 * rows * V + n}
    if op == "attend8":
        D, K, H, rows = case["dim"], case["kv_heads"], case["heads"], _rows(case)
        lens = _spread(case["lo"], case["hi"], case["batch"])
        new = rows if case["causal"] else [0] * len(rows)
        b = sum(n * 2 * K * (D + 0.25) for n, r in zip(lens, rows) if r) + sum(new) * 2 * K * 3 * D
        b += sum(rows) * H * (4 * D + 4)
        return {"bytes": int(b), "flops": 4 * D * H * sum(r * n + m * (m + 1) // 2 for n, r, m in zip(lens, rows, new))}
    held, _, _ = _pool_shape(case)
    table, n = sum(held) * 8 + len(held) * 8, _pool_pages(case)
    if op == "fork":
        return {"bytes": table + n * 8, "flops": sum(held) + n}
    if op == "reserve":
        return {"bytes": int(2 * _copied(case) * _row_bytes(case)) + table + n * 8, "flops": sum(held) + n}
    live = _pool_live(case)
    moved = live * (n - live) // n * case["page"]      # pages of any order
    return {"bytes": int(2 * moved * _row_bytes(case)) + table + n * 12, "flops": sum(held) + n}


# ------------------------------------------------------------------------------- the inputs
def _ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _fill(shape, dtype, g):
    """Normal values; those of an 8-bit cache are codes that use their type's range."""
    x = torch.empty(shape, dtype=DTYPES[dtype], device="cuda")
    flat, n = x.view(-1), 1 << 28
    for i in range(0, flat.numel(), n):
        part = torch.empty(min(n, flat.numel() - i), device="cuda").normal_(generator=g)
        flat[i:i + n] = (part.mul_(80.0).clamp_(-448.0, 448.0) if dtype == "fp8" else part).to(x.dtype)
    return x


def _scales(shape, g):
    """Powers of two: some groups of slots hold larger values than others."""
    return torch.tensor([1 / 256, 1 / 128, 1 / 64], device="cuda")[torch.randint(0, 3, shape, generator=g, device="cuda")]


def _pool_inputs(case, g):
    held, shared, width = _pool_shape(case)
    samples, page, n_pages = case["samples"], case["page"], _pool_pages(case)
    order = torch.randperm(n_pages, generator=g, device="cuda").cpu().numpy().astype(np.int32)
    table = np.zeros((len(held), width), np.int32)
    refs = np.zeros(n_pages, np.int32)
    at = 0
    for i, (h, s) in enumerate(zip(held, shared)):
        s = s if i % samples else 0
        table[i, :s] = table[i - i % samples, :s]
        table[i, s:h] = order[at:at + h - s]
        at += h - s
        np.add.at(refs, table[i, :h], 1)
    shape = (case["layers"], n_pages, case["kv_heads"], page, case["dim"])
    s = {"table": _ints(table), "held": _ints(held), "refs": _ints(refs), "lens": _ints(_pool_lens(case)),
         "k_scale": None, "v_scale": None}
    s.update(table_out=torch.zeros_like(s["table"]), held_out=torch.zeros_like(s["held"]), refs_out=torch.zeros_like(s["refs"]))
    if case["op"] != "fork":
        s["k"], s["v"] = _fill(shape, case["dtype"], g), _fill(shape, case["dtype"], g)
        if case["dtype"] == "fp8":
            s["k_scale"], s["v_scale"] = _scales(shape[:3] + (page // GROUP,), g), _scales(shape[:3] + (page // GROUP,), g)
    else:      # nothing of the pages is touched
        s["k"] = s["v"] = torch.empty(shape, dtype=DTYPES[case["dtype"]], device="cuda")
    if case["op"] == "reserve":
        s["rows"] = _ints([case["rows"] - (i % 5 == 4) for i in range(len(held))])
    if case["op"] == "fork":
        # a beam step or a scheduler's: most stay, some take another's place among the samples of the prompt, some end
        n = len(held)
        pick = torch.randint(0, samples, (n,), generator=g, device="cuda").cpu().numpy()
        b = np.arange(n)
        parent = np.where(b % 3 == 0, b, b - b % samples + pick)
        if case["keep"]:
            parent = np.where(b % 16 == 5, -1, parent)
            s["keep"] = _ints([max(0, _pool_lens(case)[p] - int(x)) if p >= 0 else 0 for p, x in zip(parent, pick)])
        s["parent"] = _ints(parent)
    return s


def _adjust_inputs(case, g):
    B, k, V = case["batch"], case["k"], case["vocab"]
    seen, prompt = _history(case)
    T = max(seen)
    logits = torch.empty((B, k + 1, V), device="cuda").normal_(generator=g) * 3.0
    s = {"logits": logits.to(DTYPES[case["dtype"]]), "lens": _ints(_drafts(case))}
    # a transcript repeats itself: tokens of a small part of the vocabulary, and the drafts of the same part
    common = torch.randint(0, V, (max(1, V // 100),), generator=g, device="cuda")
    s["history"] = common[torch.randint(0, common.numel(), (B, T), generator=g, device="cuda")].to(torch.int32)
    s["draft"] = common[torch.randint(0, min(20, common.numel()), (B, k), generator=g, device="cuda")].to(torch.int32)
    s["seen"], s["prompt"] = _ints(seen), _ints(prompt)
    s["repetition"] = 1.0 + 0.5 * torch.rand(B, generator=g, device="cuda")
    s["frequency"], s["presence"] = (torch.rand(B, generator=g, device="cuda") for _ in range(2))
    s["bias"] = s["mask"] = None
    if case["bias"]:      # a few hundred tokens preferred or suppressed, the same for all utterances
        at = torch.randint(0, V, (max(1, V // 200),), generator=g, device="cuda")
        s["bias"] = torch.zeros(V, device="cuda")
        s["bias"][at] = torch.empty(at.numel(), device="cuda").normal_(generator=g) * 5.0
        s["bias"][at[: at.numel() // 3]] = -math.inf
    if case["mask"]:      # 32 tokens a word: what a grammar's states allow, a tenth to all
        words = _ceil(V, 32)
        share = torch.rand((B, k + 1, 1, 1), generator=g, device="cuda") * 0.9 + 0.1
        bits = torch.rand((B, k + 1, words, 32), generator=g, device="cuda") < share
        s["mask"] = _pack(bits)
    s["out"] = torch.zeros_like(s["logits"])
    return s


def _pack(bits):
    w = (bits.long() << torch.arange(32, device="cuda")).sum(dim=-1)
    return torch.where(w >= 1 << 31, w - (1 << 32), w).to(torch.int32)


def _inputs(case, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    if case["op"] == "adjust":
        return _adjust_inputs(case, g)
    if case["op"] != "attend8":
        return _pool_inputs(case, g)
    B, R, H, K, D, page = (case[x] for x in ("batch", "rows", "heads", "kv_heads", "dim", "page"))
    lens, rows, causal = _spread(case["lo"], case["hi"], B), _rows(case), case["causal"]
    slots = [n + (R if causal else 0) for n in lens]
    per, need = _ceil(max(max(slots), 1), page), [_ceil(n, page) for n in slots]
    n_pages = sum(need) + 3
    # a pool in use: every sequence's pages scattered over it, a few pages free; stale values past each length
    order = torch.randperm(n_pages, generator=g, device="cuda").cpu().numpy()
    table = np.full((B, per), order[-1])
    for b, n in enumerate(need):
        table[b, :n] = order[sum(need[:b]):sum(need[:b]) + n]
    dt = DTYPES[case["dtype"]]
    s = {"k": _fill((n_pages, K, page, D), "fp8", g), "v": _fill((n_pages, K, page, D), "fp8", g),
         "k_scale": _scales((n_pages, K, page // GROUP), g), "v_scale": _scales((n_pages, K, page // GROUP), g),
         "table": _ints(table), "lens": _ints(lens), "rows": _ints(rows), "k_new": None, "v_new": None}
    # one projection's output holds the rows' queries, keys and values side by side
    qkv = torch.empty((B, R, (H + 2 * K) * D), dtype=dt, device="cuda").normal_(generator=g)
    s["q"] = qkv[:, :, :H * D].unflatten(2, (H, D))
    if causal:
        s["k_new"] = qkv[:, :, H * D:(H + K) * D].unflatten(2, (K, D))
        s["v_new"] = qkv[:, :, (H + K) * D:].unflatten(2, (K, D))
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = case
    if own:
        from paper_2608_12703_gb300 import serving
        if case["op"] == "adjust":
            s["adjust"] = serving.adjust_logits
        elif case["op"] == "attend8":
            s["cache"] = serving.PagedCache8(s["k"], s["v"], s["k_scale"], s["v_scale"], s["table"])
        else:
            caches = [serving.PagedCache(k, v, s["table"]) if s["k_scale"] is None else
                      serving.PagedCache8(k, v, s["k_scale"][i], s["v_scale"][i], s["table"])
                      for i, (k, v) in enumerate(zip(s["k"], s["v"]))]
            s["pool"] = serving.PagePool(caches, s["held"], s["refs"])
    return s


# ------------------------------------------------------------------------- the plain forms
def _codes(x):
    """8-bit values as bytes, which indexing takes."""
    return x.view(torch.uint8)


def _needed_scale(amax):
    """The least power of two (2^-126 at least) by which values of this magnitude divided are at most 448, the largest of 8 bits."""
    m, x = torch.frexp(amax)
    e = torch.where(amax > 0, torch.where(m <= 0.875, x - 9, x - 8), torch.full_like(x, -126)).clamp(min=-126)
    return ((e + 127) << 23).view(torch.float32)


def _append_plain(pages, scales, table, new, lens, rows):
    """Quantise the rows' K or V behind each sequence's slots: groups that they begin take the scale that the rows need,
    a group that goes on the larger of its own and theirs, its slots rounded anew."""
    page, (B, R, K, D) = pages.shape[2], new.shape
    groups = (R + GROUP - 2) // GROUP + 1
    base = lens.long() // GROUP * GROUP
    slot = base[:, None] + torch.arange(groups * GROUP, device="cuda")[None, :]          # [B, groups * 16]
    row = slot - lens[:, None]
    pid = table.long().gather(1, (slot // page).clamp(max=table.shape[1] - 1))
    fresh, held = (row >= 0) & (row < rows[:, None]), row < 0
    old_scale = scales[pid, :, slot % page // GROUP]                                     # [B, S, K]
    old = _codes(pages)[pid, :, slot % page].view(pages.dtype).float() * old_scale[..., None]
    x = new.float().gather(1, row.clamp(0, R - 1)[:, :, None, None].expand(-1, -1, K, D))
    x = torch.where(torch.isinf(x), math.nan, x)
    amax = torch.where(fresh[..., None, None] & ~torch.isnan(x), x.abs(), 0.0).amax(dim=3)
    need = _needed_scale(amax.unflatten(1, (groups, GROUP)).amax(dim=2))                 # [B, groups, K]
    before = torch.where(held[..., None], old_scale, 0.0).unflatten(1, (groups, GROUP)).amax(dim=2)
    scale = torch.maximum(need, before).repeat_interleave(GROUP, dim=1)
    x = torch.where(held[..., None, None], old, x)
    code = _codes((x / scale[..., None]).to(pages.dtype))
    use = (fresh | held) & (rows > 0)[:, None]
    _codes(pages)[pid[use], :, (slot % page)[use]] = code[use]
    scales[pid[use], :, (slot % page // GROUP)[use]] = scale[use]


def _gather8(pages, scales, table, n):
    """[B, K, n, D] of the sequences' first n slots, dequantised."""
    x = _codes(pages)[table.long()].view(pages.dtype).float() * scales[table.long()].repeat_interleave(GROUP, dim=3)[..., None]
    return x.transpose(1, 2).flatten(2, 3)[:, :, :n]


def _attend8_plain(case, s):
    B, R, H, K, D = (case[x] for x in ("batch", "rows", "heads", "kv_heads", "dim"))
    causal, G = case["causal"], H // K
    if causal:
        _append_plain(s["k"], s["k_scale"], s["table"], s["k_new"], s["lens"], s["rows"])
        _append_plain(s["v"], s["v_scale"], s["table"], s["v_new"], s["lens"], s["rows"])
    out = torch.empty((B, R, H, D), dtype=s["q"].dtype, device="cuda")
    lse = torch.empty((B, R, H), device="cuda")
    most = s["table"].shape[1] * case["page"]
    step = max(1, int(3e8 // ((K * D + H * R) * most)))
    slot, row = torch.arange(most, device="cuda"), torch.arange(R, device="cuda")[:, None]
    for b in range(0, B, step):
        t, n, r = s["table"][b:b + step], s["lens"][b:b + step, None, None, None], s["rows"][b:b + step, None, None, None]
        k, v = _gather8(s["k"], s["k_scale"], t, most), _gather8(s["v"], s["v_scale"], t, most)
        q = s["q"][b:b + step].float().permute(0, 2, 1, 3).reshape(-1, K, G * R, D)
        x = (q @ k.transpose(2, 3) * (1.0 / math.sqrt(D))).reshape(-1, H, R, most)
        x = x.masked_fill((slot >= n + (row + 1 if causal else 0)) | (row >= r), -math.inf)
        v = torch.where(slot[:, None] < n + (r if causal else 0), v, 0.0)
        m = x.amax(dim=-1, keepdim=True)
        e = torch.exp(x - torch.where(torch.isinf(m), 0.0, m))
        l = e.sum(dim=-1, keepdim=True)
        o = (e.reshape(-1, K, G * R, most) @ v).reshape(-1, H, R, D) / torch.where(l > 0, l, 1.0)
        out[b:b + step] = o.permute(0, 2, 1, 3).to(out.dtype)
        lse[b:b + step] = (m + torch.log(l)).squeeze(-1).permute(0, 2, 1)
    return out, lse, s["k"], s["v"], s["k_scale"], s["v_scale"]


def _count(refs, ids, by):
    refs.index_add_(0, ids.long(), torch.full_like(ids, by))


def _reserve_plain(case, s):
    table, held, refs, lens, rows, page = s["table"], s["held"], s["refs"], s["lens"], s["rows"], case["page"]
    B, W = table.shape
    j = torch.arange(W, device="cuda")[None, :]
    first, last = (lens // page)[:, None], ((lens + rows - 1) // page)[:, None]
    touched = (rows > 0)[:, None] & (j >= first) & (j <= last)
    have = j < held[:, None]
    shared = touched & have & (refs[torch.where(have, table, 0).long()] > 1)
    # of the sequences whose last page only they share the lowest keeps it
    b = torch.arange(B, device="cuda", dtype=torch.int32)[:, None].expand(B, W)
    tail = shared & (j == first)
    holders, lowest = torch.zeros_like(refs), torch.full_like(refs, B)
    _count(holders, table[tail], 1)
    lowest.scatter_reduce_(0, table[tail].long(), b[tail], "amin")
    at = torch.where(have, table, 0).long()
    fresh = (touched & ~have) | (shared & ~(tail & (holders[at] == refs[at]) & (lowest[at] == b)))
    free = torch.nonzero(refs == 0).flatten().to(torch.int32)
    rank = torch.cumsum(fresh.flatten().long(), 0).reshape(B, W)
    need = int(rank[-1, -1])
    counts = torch.tensor([need, free.numel() - need], dtype=torch.int32)
    if need > free.numel():
        fresh, need, counts = torch.zeros_like(fresh), 0, torch.tensor([0, free.numel()], dtype=torch.int32)
        last = held[:, None] - 1
    ids = free[:need]
    held_out = torch.where(rows > 0, torch.maximum(held, last[:, 0] + 1), held)
    old = table[fresh & have]
    new = table.clone()
    new[fresh] = ids
    s["table_out"] = torch.where(j < held_out[:, None], new, s["table_out"])
    s["held_out"], s["refs_out"] = held_out, refs.clone()
    _count(s["refs_out"], old, -1)
    _count(s["refs_out"], ids, 1)
    copy = fresh & have & (j == first)
    n = (lens % page)[:, None].expand(B, W)[copy][:, None]
    src, dst = table[copy].long(), new[copy].long()
    if src.numel():
        use = (torch.arange(page, device="cuda") < n)[:, None, :, None]
        used = (torch.arange(page // GROUP, device="cuda") * GROUP < n)[:, None]
        for p in (s["k"], s["v"]):
            p = _codes(p) if case["dtype"] == "fp8" else p
            p[:, dst] = torch.where(use, p[:, src], p[:, dst])
        for p in (s["k_scale"], s["v_scale"]):
            if p is not None:
                p[:, dst] = torch.where(used, p[:, src], p[:, dst])
    return [s["table_out"], s["held_out"], s["refs_out"], counts] + _pages(s)


def _pages(s):
    return [s["k"], s["v"]] + ([] if s["k_scale"] is None else [s["k_scale"], s["v_scale"]])


def _fork_plain(case, s):
    table, held, page = s["table"], s["held"], case["page"]
    j = torch.arange(table.shape[1], device="cuda")[None, :]
    p = s["parent"].clamp(min=0).long()
    n = held[p]
    if case["keep"]:
        n = torch.minimum(n, (s["keep"] + page - 1) // page)
    n = torch.where(s["parent"] < 0, 0, n)
    use, new = j < n[:, None], table[p]
    refs = s["refs"].clone()
    _count(refs, table[j < held[:, None]], -1)
    _count(refs, new[use], 1)
    s["table_out"], s["held_out"], s["refs_out"] = torch.where(use, new, s["table_out"]), n, refs
    return s["table_out"], s["held_out"], s["refs_out"]


def _compact_plain(case, s):
    refs, table = s["refs"], s["table"]
    used = refs > 0
    ids = torch.arange(refs.numel(), device="cuda", dtype=torch.int32)
    live = used.sum().to(torch.int32)
    src, dst = torch.nonzero(used & (ids >= live)).flatten(), torch.nonzero(~used & (ids < live)).flatten()
    where = torch.where(used, ids, -1)
    where[src] = dst.to(torch.int32)
    s["refs_out"] = torch.where(ids < live, refs, 0)
    s["refs_out"][dst] = refs[src]
    use = torch.arange(table.shape[1], device="cuda")[None, :] < s["held"][:, None]
    s["table_out"] = torch.where(use, where[torch.where(use, table, 0).long()], s["table_out"])
    for p in _pages(s):
        p = _codes(p) if p.dtype == torch.float8_e4m3fn else p
        p[:, dst] = p[:, src]
    return [s["table_out"], s["refs_out"], where, live.reshape(1)] + _pages(s)


def _adjust_plain(case, s):
    B, R, V = s["logits"].shape
    at = torch.arange(s["history"].shape[1], device="cuda")[None, :]
    live = at < s["seen"][:, None]
    # tokens seen before row 0, those of the transcript alone, and what the rows' own drafts add
    every = torch.zeros((B, 1, V), device="cuda").scatter_add_(2, s["history"].long()[:, None], live[:, None].float())
    said = torch.zeros((B, 1, V), device="cuda").scatter_add_(2, s["history"].long()[:, None],
                                                              (live & (at >= s["prompt"][:, None]))[:, None].float())
    drafted = torch.zeros((B, R, V), device="cuda")
    if R > 1:
        drafted[:, 1:].scatter_(2, s["draft"].long()[..., None], 1.0)
        drafted = torch.cumsum(drafted, dim=1)
    count, seen = said + drafted, every + drafted > 0
    x, rep = s["logits"].float(), s["repetition"][:, None, None]
    x = torch.where(seen, torch.where(x > 0, x / rep, x * rep), x)
    x = x - s["frequency"][:, None, None] * count - s["presence"][:, None, None] * (count > 0)
    if s["bias"] is not None:
        x = x + s["bias"]
    if s["mask"] is not None:
        v = torch.arange(V, device="cuda")
        x = torch.where((s["mask"][..., v // 32] >> (v % 32)) & 1 > 0, x, -math.inf)
    use = (torch.arange(R, device="cuda")[None, :] <= s["lens"][:, None])[..., None]
    s["out"] = torch.where(use, x.to(s["out"].dtype), s["out"])
    return s["out"]


def run(s):
    case = s["case"]
    op = case["op"]
    if not own:
        return {"attend8": _attend8_plain, "reserve": _reserve_plain, "fork": _fork_plain, "compact": _compact_plain,
                "adjust": _adjust_plain}[op](case, s)
    if op == "attend8":
        out, lse = s["cache"].attend(s["q"], s["lens"], k_new=s["k_new"], v_new=s["v_new"], rows=s["rows"], causal=case["causal"])
        return out, lse, s["k"], s["v"], s["k_scale"], s["v_scale"]
    if op == "adjust":
        return s["adjust"](s["logits"], history=s["history"], history_len=s["seen"], prompt_len=s["prompt"], draft=s["draft"],
                           lens=s["lens"], repetition=s["repetition"], frequency=s["frequency"], presence=s["presence"],
                           bias=s["bias"], mask=s["mask"], out=s["out"])
    pool, to = s["pool"], dict(table_out=s["table_out"], refs_out=s["refs_out"])
    if op == "compact":
        return list(pool.compact(**to)) + _pages(s)
    if op == "fork":
        return pool.fork(s["parent"], s.get("keep"), held_out=s["held_out"], **to)
    return list(pool.reserve(s["lens"], s["rows"], held_out=s["held_out"], **to)) + _pages(s)


# --------------------------------------------------------- the definition in 64 bits
def exact(case, seed):
    s = _inputs(case, seed)
    op = case["op"]
    if op == "adjust":
        return _adjust_exact(case, s)
    if op == "fork":
        return _fork_exact(case, s)
    if op == "reserve":
        return _reserve_exact(case, s)
    if op == "compact":
        return _compact_exact(case, s)
    if work(case)["flops"] > 2e11 or s["k"].numel() > 3e9:
        return None
    return _attend8_exact(case, s)


def _store(pages, scales, row, new, n, page):
    """Quantise new [r, K, D] into slots n .. of the sequence whose pages are `row`, one group at a time, all heads together."""
    r = new.shape[0]
    for g in range(n // GROUP, (n + r - 1) // GROUP + 1):
        pid, at = row[g * GROUP // page], g * GROUP % page
        a, b = max(n, g * GROUP), min(n + r, (g + 1) * GROUP)
        x = new[a - n:b - n].double()
        need = x.abs().amax(dim=(0, 2))
        scale = torch.exp2(torch.ceil(torch.log2(need / 448.0)).clamp(min=-126.0))
        # log2 may be off by a rounding: the least power of two that does
        scale = torch.where(scale * 448.0 < need, scale * 2, torch.where(scale * 224.0 >= need, scale / 2, scale)).clamp(min=2.0 ** -126)
        kept = a - g * GROUP
        x = x.transpose(0, 1)
        if kept:
            was = scales[pid, :, at // GROUP].double()
            scale = torch.maximum(scale, was)
            x = torch.cat([pages[pid, :, at:at + kept].float().double() * was[:, None, None], x], dim=1)
        pages[pid, :, at:at + x.shape[1]] = (x / scale[:, None, None]).float().to(pages.dtype)
        scales[pid, :, at // GROUP] = scale.float()


def _attend8_exact(case, s):
    B, R, H, K, D, page = (case[x] for x in ("batch", "rows", "heads", "kv_heads", "dim", "page"))
    lens, rows, causal, G = _spread(case["lo"], case["hi"], B), _rows(case), case["causal"], H // K
    table = s["table"].cpu().tolist()
    out = torch.zeros((B, R, H, D), dtype=torch.float64, device="cuda")
    lse = torch.full((B, R, H), -math.inf, dtype=torch.float64, device="cuda")
    for b in range(B):
        n, r = lens[b], rows[b]
        if causal and r:
            _store(s["k"], s["k_scale"], table[b], s["k_new"][b, :r], n, page)
            _store(s["v"], s["v_scale"], table[b], s["v_new"][b, :r], n, page)
        end = n + (r if causal else 0)
        if not r or not end:
            continue

        def walk(pages, scales):
            ids = table[b][:_ceil(end, page)]
            x = torch.stack([pages[i].float() for i in ids]).double()
            x = x.unflatten(2, (page // GROUP, GROUP)) * torch.stack([scales[i] for i in ids]).double()[..., None, None]
            return x.flatten(2, 3).transpose(0, 1).flatten(1, 2)[:, :end]

        k, v = walk(s["k"], s["k_scale"]), walk(s["v"], s["v_scale"])
        for h in range(H):
            x = s["q"][b, :r, h].double() @ k[h // G].T / math.sqrt(D)
            if causal:
                x = x.masked_fill(torch.ones_like(x, dtype=torch.bool).triu(n + 1), -math.inf)
            lse[b, :r, h] = torch.logsumexp(x, 1)
            out[b, :r, h] = torch.softmax(x, 1) @ v[h // G]
    return out, lse, s["k"], s["v"], s["k_scale"], s["v_scale"]


def _reserve_exact(case, s):
    """One sequence at a time, on the host."""
    table, held, refs = (s[x].cpu().numpy().copy() for x in ("table", "held", "refs"))
    lens, rows, page = s["lens"].cpu().tolist(), s["rows"].cpu().tolist(), case["page"]
    free = [int(i) for i in np.flatnonzero(refs == 0)]
    was, taken, by_page = refs.copy(), 0, {}
    for b, (n, r) in enumerate(zip(lens, rows)):
        if r and n // page < held[b]:
            by_page.setdefault(int(table[b, n // page]), []).append(b)
    for b, (n, r) in enumerate(zip(lens, rows)):
        for j in range(n // page, (n + r - 1) // page + 1 if r else 0):
            if j < held[b]:
                old = int(table[b, j])
                if was[old] <= 1 or (j == n // page and len(by_page[old]) == was[old] and by_page[old][0] == b):
                    continue
                refs[old] -= 1
            new = free[taken]
            taken += 1
            refs[new] += 1
            if j < held[b] and j == n // page and n % page:
                m = n % page
                for p in (s["k"], s["v"]):
                    p[:, new, :, :m] = p[:, old, :, :m]
                for p in (s["k_scale"], s["v_scale"]):
                    if p is not None:
                        p[:, new, :, :_ceil(m, GROUP)] = p[:, old, :, :_ceil(m, GROUP)]
            table[b, j] = new
        if r:
            held[b] = max(held[b], (n + r - 1) // page + 1)
    out = s["table_out"].cpu().numpy()
    for b in range(len(held)):
        out[b, :held[b]] = table[b, :held[b]]
    counts = torch.tensor([taken, len(free) - taken], dtype=torch.int32)
    return [torch.from_numpy(out), torch.from_numpy(held), torch.from_numpy(refs), counts] + _pages(s)


def _fork_exact(case, s):
    table, held, refs = (s[x].cpu().numpy() for x in ("table", "held", "refs"))
    out, n_out = s["table_out"].cpu().numpy(), held.copy()
    refs = np.zeros_like(refs)
    for b, p in enumerate(s["parent"].cpu().tolist()):
        n = 0 if p < 0 else int(held[p])
        if case["keep"]:
            n = min(n, _ceil(int(s["keep"][b]), case["page"]))
        out[b, :n], n_out[b] = table[p, :n], n
        np.add.at(refs, out[b, :n], 1)
    return torch.from_numpy(out), torch.from_numpy(n_out), torch.from_numpy(refs)


def _compact_exact(case, s):
    table, held, refs = (s[x].cpu().numpy() for x in ("table", "held", "refs"))
    live = int((refs > 0).sum())
    dst, src = np.flatnonzero(refs[:live] == 0), live + np.flatnonzero(refs[live:] > 0)
    where = np.where(refs > 0, np.arange(refs.size), -1).astype(np.int32)
    where[src] = dst
    refs_out, out = np.zeros_like(refs), s["table_out"].cpu().numpy()
    for old, new in enumerate(where):
        if new >= 0:
            refs_out[new] = refs[old]
    for b, h in enumerate(held):
        out[b, :h] = where[table[b, :h]]
    for p in _pages(s):
        for a, b in zip(dst, src):
            p[:, int(a)] = p[:, int(b)]
    return [torch.from_numpy(out), torch.from_numpy(refs_out), torch.from_numpy(where), torch.tensor([live], dtype=torch.int32)] + _pages(s)


def _adjust_exact(case, s):
    """One row at a time."""
    B, R, V = s["logits"].shape
    out = s["out"].double()
    seen, prompt = _history(case)
    rep, freq, pres = (s[x].double().tolist() for x in ("repetition", "frequency", "presence"))
    for b, n in enumerate(_drafts(case)):
        for i in range(n + 1):
            said = torch.cat([s["history"][b, prompt[b]:seen[b]], s["draft"][b, :i]]).long()
            before = torch.cat([s["history"][b, :prompt[b]].long(), said])
            count = torch.bincount(said, minlength=V).double()
            x = s["logits"][b, i].double()
            x[before] = torch.where(x[before] > 0, x[before] / rep[b], x[before] * rep[b])
            x -= freq[b] * count
            x[count > 0] -= pres[b]
            if s["bias"] is not None:
                x += s["bias"].double()
            if s["mask"] is not None:
                bits = np.unpackbits(s["mask"][b, i].cpu().numpy().view(np.uint8), bitorder="little")[:V]
                x[torch.from_numpy(bits == 0).cuda()] = -math.inf
            out[b, i] = x
    return out
