"""Rounds of a serving loop with several samples a prompt over an 8-bit cache: fork, private pages, attention with append,
adjusted logits, sampled acceptance, pages of rejected drafts given back, compaction now and then.  Every step against the
plain implementations on a copy of the state."""
import math

import numpy as np
import pytest
import torch

import cache8_ref as ref
import serving_ref
from paper_2608_12703_gb300 import asrspec as A
from test_gpu_cache8 import codes, compare, i32, same_bits

pytestmark = pytest.mark.gpu

LAYERS, K, H, D, V, PAGE, DRAFTS, WIDTH = 2, 2, 4, 64, 517, 16, 4, 12


def host(x):
    return x.cpu().numpy().astype(np.int64)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_rounds(built_lib, cuda, dtype):
    from paper_2608_12703_gb300 import serving
    g = torch.Generator(device="cuda").manual_seed(5)
    rng = np.random.default_rng(5)
    B, prompts, n_pages = 6, [37, 52], 60

    def randn(*shape):
        return torch.randn(shape, generator=g, device="cuda")

    table = torch.zeros((B, WIDTH), dtype=torch.int32, device="cuda")
    held, refs = torch.zeros(B, dtype=torch.int32, device="cuda"), torch.zeros(n_pages, dtype=torch.int32, device="cuda")
    layers = []
    for _ in range(LAYERS):
        k, v = (torch.full((n_pages, K, PAGE, D), 0x7f, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn) for _ in range(2))
        ks, vs = (torch.full((n_pages, K, 1), math.nan, device="cuda") for _ in range(2))
        layers.append((k, v, ks, vs))
    caches = [serving.PagedCache8(*x, table) for x in layers]
    pool = serving.PagePool(caches, held, refs)

    def attend(lens, rows, R):
        """New rows in every layer, against the same on copies of the pages."""
        n = i32(lens)
        for cache, (k, v, ks, vs) in zip(caches, layers):
            q, kn, vn = (randn(B, R, h, D).to(dtype) for h in (H, K, K))
            kr, vr, ksr, vsr = k.clone(), v.clone(), ks.clone(), vs.clone()
            ref.append(kr, ksr, table, lens, rows, kn)
            ref.append(vr, vsr, table, lens, rows, vn)
            out, lse = cache.attend(q, n, k_new=kn, v_new=vn, rows=i32(rows))
            assert cache.status() == 0
            assert torch.equal(codes(k), codes(kr)) and torch.equal(codes(v), codes(vr)) and same_bits(ks, ksr) and same_bits(vs, vsr)
            compare(out, lse, *ref.attend(q, kr, vr, ksr, vsr, table, lens, rows, True, 1 / math.sqrt(D)))

    def checked(got, want):
        table_w, held_w, refs_w = want
        for b in range(B):
            assert host(table)[b, :held_w[b]].tolist() == list(table_w[b, :held_w[b]])
        assert host(held).tolist() == list(held_w) and host(refs).tolist() == list(refs_w)
        assert got[0] is table and pool.status() == 0

    def reserve(lens, rows):
        want = ref.reserve(host(table), host(held), host(refs), lens, rows, PAGE)
        got = pool.reserve(i32(lens), i32(rows))
        checked(got, want[:3])
        assert got[3].tolist() == list(want[3])

    # the prompts, in the first sample of each; the others go on from them
    lens, rows = [0] * B, [prompts[b // 3] if b % 3 == 0 else 0 for b in range(B)]
    reserve(lens, rows)
    attend(lens, rows, max(rows))
    parent = [b - b % 3 for b in range(B)]
    want = ref.fork(host(table), host(held), host(refs), parent, None, PAGE)
    checked(pool.fork(i32(parent)), want)
    assert int(refs.max()) == 3
    lens = [prompts[b // 3] for b in range(B)]
    seen = [list(rng.integers(0, V, n)) for n in (prompts[b // 3] for b in range(B))]

    for turn in range(5):
        drafts = [int(x) for x in rng.integers(0, DRAFTS + 1, B)]
        rows = [n + 1 for n in drafts]
        if turn == 3:
            drafts[2], rows[2] = -1, 0      # sits out
        reserve(lens, rows)
        attend(lens, rows, DRAFTS + 1)
        # logits that repeat what was said, a grammar that allows a third
        T = max(len(s) for s in seen)
        history = np.zeros((B, T), np.int32)
        for b, s in enumerate(seen):
            history[b, :len(s)] = s
        draft = rng.integers(0, V, (B, DRAFTS)).astype(np.int32)
        mask = (rng.integers(-2 ** 31, 2 ** 31, (B, DRAFTS + 1, -(-V // 32))) & rng.integers(-2 ** 31, 2 ** 31, (B, DRAFTS + 1, -(-V // 32)))
                | 1).astype(np.int32)
        logits = randn(B, DRAFTS + 1, V) * 3
        rep, freq, pres = np.float32(1.3), np.float32(0.2), np.float32(0.1)
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        args = dict(history=i32(history.ravel()).reshape(B, T), history_len=i32([len(s) for s in seen]), prompt_len=i32([prompts[b // 3] for b in range(B)]),
                    draft=i32(draft.ravel()).reshape(B, DRAFTS), lens=i32(drafts), mask=torch.tensor(mask, device="cuda"))
        before = logits.cpu().numpy()
        adjusted = serving.adjust_logits(logits, repetition=float(rep), frequency=float(freq), presence=float(pres), status=status, **args)
        want, bound = ref.adjust(before, history, [len(s) for s in seen], [prompts[b // 3] for b in range(B)], draft, drafts, [rep] * B,
                                 [freq] * B, [pres] * B, None, mask)
        fin = np.isfinite(want)
        assert (np.abs(adjusted.double().cpu().numpy()[fin] - want[fin]) <= 1.01 * bound[fin]).all()
        u, race = torch.rand((B, DRAFTS), generator=g, device="cuda"), -torch.log(torch.rand((B, V), generator=g, device="cuda"))
        accepted, token, step, _ = serving.accept_sampled(adjusted, args["draft"], args["lens"], u, race, status=status)
        wa, wt, ws, _, margin = serving_ref.accept(adjusted.cpu().numpy(), draft, drafts, u.cpu().numpy(), race.cpu().numpy(), None, 1.0)
        sure = margin > 1e-4
        assert int(status) == 0 and (host(accepted)[sure] == wa[sure]).all() and (host(token)[sure] == wt[sure]).all()
        for b in range(B):
            if drafts[b] < 0:
                assert int(step[b]) == 0
                continue
            n, t = int(accepted[b]), int(token[b])
            assert int(step[b]) == n + 1 and (mask[b, n, t // 32] >> (t % 32)) & 1
            seen[b] += list(draft[b, :n]) + [t]
            lens[b] += n + 1
        # samples change places; the pages behind rejected drafts go back
        parent = [b - b % 3 + int(rng.integers(0, 3)) if b % 2 else b for b in range(B)]
        keep = [lens[p] for p in parent]
        want = ref.fork(host(table), host(held), host(refs), parent, keep, PAGE)
        checked(pool.fork(i32(parent), i32(keep)), want)
        lens, seen = keep, [list(seen[p]) for p in parent]
        if turn % 2:
            old = [[x.clone() for x in layer] for layer in layers]
            table_w, refs_w, where, live, moves = ref.compact(host(table), host(held), host(refs))
            got = pool.compact()
            checked(got, (table_w, host(held), refs_w))
            assert host(got[2]).tolist() == where.tolist() and int(got[3]) == live
            for layer, was in zip(layers, old):
                for x, y in zip(layer, was):
                    for a, b in moves:
                        y[b] = y[a].clone()
                    assert same_bits(x, y)
    assert pool.status() == 0 and all(c.status() == 0 for c in caches) and A.ST_CAPACITY == 4
