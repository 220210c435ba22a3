"""Sampled speculative decoding over a bounded paged cache, end to end.

A small random-weight decoder is the target, its embedding and head alone the draft.  One
round per sequence: the draft draws k tokens; the target scores the pending
token and the drafts in one pass, appending their K/V to the pages
(``PagedCache.attend``); ``accept_sampled`` keeps the drafts that the target's
probabilities allow and draws the next token; ``PagedCache.weigh`` credits the
cached slots with the attention of the committed rows; and every few rounds
``PagedCache.evict`` cuts every head to its most attended slots, so the cache
never grows past its pages however long the transcript gets.

    python examples/paged_sampling.py [--rounds 200] [--batch 8] [--drafts 4] [--budget 256]
"""
from __future__ import annotations

import argparse
import os
import sys
import time

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2608_12703_gb300 import serving  # noqa: E402


class Model:
    """Random weights of a pre-norm decoder: shared K/V heads, sinusoidal positions."""

    def __init__(self, layers, heads, kv_heads, head_dim, vocab, dtype, seed=0):
        g = torch.Generator().manual_seed(seed)
        d = heads * head_dim
        self.layers, self.heads, self.kv_heads, self.head_dim, self.vocab, self.dtype, self.d = (
            layers, heads, kv_heads, head_dim, vocab, dtype, d)

        def w(*shape):
            return (torch.randn(shape, generator=g) / shape[-1] ** 0.5).to("cuda", dtype)
        self.emb, self.head = w(vocab, d) * d ** 0.5, w(vocab, d) * 2
        self.qkv = [w((heads + 2 * kv_heads) * head_dim, d) for _ in range(layers)]
        self.out = [w(d, d) * 0.5 for _ in range(layers)]
        self.up = [w(2 * d, d) for _ in range(layers)]
        self.down = [w(d, 2 * d) * 0.5 for _ in range(layers)]
        self.freq = torch.exp(-torch.arange(0, d, 2, device="cuda") / d * 9.0)

    def positions(self, pos):
        a = pos[..., None].float() * self.freq
        return torch.cat([torch.sin(a), torch.cos(a)], dim=-1).to(self.dtype)


def norm(x):
    return torch.nn.functional.layer_norm(x.float(), x.shape[-1:]).to(x.dtype)


class Decoder:
    """The state of a batch: per layer a pool of pages, accumulated weights and the slots' positions; lengths shared by
    the layers (every layer keeps the same number of slots)."""

    def __init__(self, model, batch, drafts, budget, evict_every=8, recent=16, page=32, temperature=1.0, seed=1,
                 cache=serving.PagedCache, accept=serving.accept_sampled):
        m, self.m = model, model
        self.B, self.k, self.budget, self.evict_every, self.recent = batch, drafts, budget, evict_every, recent
        self.temperature, self.accept = temperature, accept
        slots = budget + (evict_every + 1) * (drafts + 1)
        per = -(-slots // page)
        table = torch.randperm(batch * per, device="cuda").to(torch.int32).view(batch, per)
        shape = (batch * per, m.kv_heads, page, m.head_dim)
        self.caches = [cache(torch.zeros(shape, dtype=m.dtype, device="cuda"), torch.zeros(shape, dtype=m.dtype, device="cuda"),
                             table) for _ in range(m.layers)]
        self.score = [torch.zeros((batch, m.kv_heads, per * page), device="cuda") for _ in range(m.layers)]
        self.pos = [torch.zeros((batch, m.kv_heads, per * page), dtype=torch.int32, device="cuda") for _ in range(m.layers)]
        self.kv_len = torch.zeros(batch, dtype=torch.int32, device="cuda")
        self.seen = torch.zeros(batch, dtype=torch.int32, device="cuda")
        self.pending = torch.arange(batch, device="cuda") % m.vocab
        self.g = torch.Generator(device="cuda").manual_seed(seed)
        self.rounds = 0

    def _exponential(self, *shape):
        return torch.empty(shape, device="cuda").exponential_(generator=self.g).clamp_(min=1e-30)

    def draft(self):
        tokens, logits, t = [], [], self.pending
        for _ in range(self.k):
            q = norm(self.m.emb[t]) @ self.m.head.T
            logits.append(q)
            t = (torch.log_softmax(q.float() / self.temperature, -1) - self._exponential(self.B, self.m.vocab).log()).argmax(-1)
            tokens.append(t)
        return torch.stack(tokens, 1), torch.stack(logits, 1)

    def score_rows(self, tokens):
        """Logits of the rows [B, k + 1], their K/V appended; keeps what ``weigh`` needs."""
        m, (B, R) = self.m, tokens.shape
        x = m.emb[tokens] + m.positions(self.seen[:, None] + torch.arange(R, device="cuda"))
        kept = []
        for i, c in enumerate(self.caches):
            qkv = (norm(x) @ m.qkv[i].T).view(B, R, m.heads + 2 * m.kv_heads, m.head_dim)
            q, k, v = qkv.split([m.heads, m.kv_heads, m.kv_heads], dim=2)
            o, lse = c.attend(q, self.kv_len, k_new=k, v_new=v)
            kept.append((q, lse))
            x = x + o.reshape(B, R, m.d) @ m.out[i].T
            x = x + torch.nn.functional.gelu(norm(x) @ m.up[i].T) @ m.down[i].T
        return norm(x) @ m.head.T, kept

    def round(self):
        """One round; returns (drafts [B, k], accepted [B], token [B])."""
        tokens, q = self.draft()
        target, kept = self.score_rows(torch.cat([self.pending[:, None], tokens], 1))
        drafts = tokens.to(torch.int32)
        u = torch.rand((self.B, self.k), generator=self.g, device="cuda")
        accepted, token, step, _ = self.accept(target, drafts, None, u, self._exponential(self.B, self.m.vocab),
                                               draft_logits=q, temperature=self.temperature)
        for c, (qi, lse), score, pos in zip(self.caches, kept, self.score, self.pos):
            c.weigh(qi, lse, self.kv_len, score, rows=step, pos=pos, first_pos=self.seen)
        self.kv_len = self.kv_len + step
        self.seen = self.seen + step
        self.pending = token.long()
        self.rounds += 1
        if self.rounds % self.evict_every == 0:
            for c, score, pos in zip(self.caches, self.score, self.pos):
                lens, _, _ = c.evict(self.kv_len, score, pos, self.seen, budget=self.budget, recent=self.recent, first=1)
            self.kv_len = lens
        return drafts, accepted, token


def main():
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--rounds", type=int, default=200)
    ap.add_argument("--batch", type=int, default=8)
    ap.add_argument("--drafts", type=int, default=4)
    ap.add_argument("--budget", type=int, default=256)
    a = ap.parse_args()
    dec = Decoder(Model(4, 8, 4, 64, 2000, torch.bfloat16), a.batch, a.drafts, a.budget)
    for _ in range(3):
        dec.round()
    torch.cuda.synchronize()
    seen0, t0 = dec.seen.clone(), time.perf_counter()
    accepted = torch.zeros(a.batch, device="cuda")
    for _ in range(a.rounds):
        accepted += dec.round()[1]
    torch.cuda.synchronize()
    dt = time.perf_counter() - t0
    n = int((dec.seen - seen0).sum())
    assert all(c.status() == 0 for c in dec.caches)
    print(f"{n} tokens in {dt:.3f} s ({n / dt:.0f} tokens/s), {float(accepted.mean()) / a.rounds:.2f} of {a.drafts} drafts "
          f"accepted a round, {int(dec.seen.max())} tokens seen, {int(dec.kv_len.max())} slots held")


if __name__ == "__main__":
    main()
