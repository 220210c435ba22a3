"""The example's decode loop with the library's operators against the same loop
with plain 64-bit ones: the same tokens, lengths and slots, over evictions."""
import os
import sys

import pytest
import torch

import serving_ref as ref

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))

pytestmark = pytest.mark.gpu


class PlainCache:
    """The paged operators in 64 bits, results rounded to the tensors' types."""

    def __init__(self, k_pages, v_pages, table):
        self.k, self.v, self.table = k_pages, v_pages, table

    def attend(self, q, kv_len, *, k_new, v_new):
        rows = [q.shape[1]] * q.shape[0]
        out, lse, _, _ = ref.attend(q, self.k, self.v, self.table, kv_len, rows, k_new, v_new, True, q.shape[3] ** -0.5)
        return out.to(q.dtype), lse.float()

    def weigh(self, q, lse, kv_len, score, *, rows, pos, first_pos):
        new, _ = ref.weigh(q, lse, self.k, self.table, kv_len, rows, score, True, q.shape[3] ** -0.5)
        live = ~torch.isnan(new)
        score[live] = new[live].float()
        for b in range(q.shape[0]):
            for i in range(int(rows[b])):
                pos[b, :, int(kv_len[b]) + i] = int(first_pos[b]) + i

    def evict(self, lens, score, pos, seen, *, budget, recent, first):
        plan = ref.evict(lens, score.cpu(), pos.cpu(), seen, budget, recent, first)
        page = self.k.shape[2]
        for b in range(score.shape[0]):
            for h in range(score.shape[1]):
                order = torch.tensor(plan[b][h], dtype=torch.long, device="cuda")
                m = len(order)
                at, of = self.table[b].long()[torch.arange(m, device="cuda") // page], self.table[b].long()[order // page]
                to = torch.arange(m, device="cuda") % page
                for x in (self.k, self.v):
                    x[at, h, to] = x[of, h, order % page].clone()
                score[b, h, :m], pos[b, h, :m] = score[b, h][order].clone(), pos[b, h][order].clone()
        return lens.clamp(max=budget), score, pos


def plain_accept(target, draft, lens, u, race, *, draft_logits, temperature):
    n = torch.full((target.shape[0],), draft.shape[1]).numpy()
    acc, tok, step, prob, margin = ref.accept(target.double().cpu().numpy(), draft.cpu().numpy(), n, u.double().cpu().numpy(),
                                              race.cpu().numpy(), draft_logits.double().cpu().numpy(), temperature)
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
    return i32(acc), i32(tok), i32(step), torch.tensor(prob, device="cuda")


def test_decode_loop_matches_plain_operators(built_lib, cuda):
    import paged_sampling as ex
    args = dict(batch=3, drafts=3, budget=24, evict_every=3, recent=4, page=16)
    torch.manual_seed(0)
    model = ex.Model(2, 4, 2, 64, 300, torch.float32)
    ours = ex.Decoder(model, **args)
    plain = ex.Decoder(model, cache=PlainCache, accept=plain_accept, **args)
    taken = 0
    for _ in range(20):
        a, b = ours.round(), plain.round()
        assert all(torch.equal(x, y) for x, y in zip(a, b))
        assert torch.equal(ours.kv_len, plain.kv_len) and torch.equal(ours.seen, plain.seen)
        for x, y, n in zip(ours.pos, plain.pos, range(2)):
            for i, m in enumerate(ours.kv_len.tolist()):
                assert torch.equal(x[i, :, :m], y[i, :, :m])
        taken += int(a[1].sum())
    assert all(c.status() == 0 for c in ours.caches)
    assert int(ours.seen.min()) > 24 and int(ours.kv_len.max()) <= 24 + 3 * 4 and taken > 0


def test_example_runs_in_16_bits(built_lib, cuda):
    import paged_sampling as ex
    dec = ex.Decoder(ex.Model(2, 8, 4, 64, 500, torch.bfloat16), batch=5, drafts=4, budget=64, evict_every=4)
    for _ in range(24):
        _, accepted, token = dec.round()
        assert bool(((accepted >= 0) & (accepted <= 4)).all()) and bool(((token >= 0) & (token < 500)).all())
    assert all(c.status() == 0 for c in dec.caches)
    assert int(dec.kv_len.max()) <= 64 + 4 * 5
