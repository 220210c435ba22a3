"""Rows of q that hold an infinity come out as NaN wherever they see a slot, also where every score that they see is -inf; rows
beside them, and rows that see nothing, are as they would be."""
import math

import pytest
import torch

import cache8_ref as ref
from test_gpu_cache8 import DT, compare, fill, gen, i32, make_rows, pool, same_bits

pytestmark = pytest.mark.gpu


def attend(dtype, dim, heads, kv_heads, R, lens, rows, causal, spoil):
    from paper_2608_12703_gb300 import serving
    g, page = gen(50), 32
    k, v, ks, vs, table = pool(g, kv_heads, dim, page, [n + R for n in lens])
    fill(g, k, ks, table, [n + R for n in lens])
    fill(g, v, vs, table, [n + R for n in lens])
    q = make_rows(g, len(lens), R, heads, kv_heads, dim, DT[dtype], True)[0]
    spoiled = spoil(q, k, table)      # rows [b, i, h] that hold an infinity
    c = serving.PagedCache8(k, v, ks, vs, table)
    out, lse = c.attend(q, i32(lens), rows=i32(rows), causal=causal)
    assert c.status() == 0
    clean = q.clone()
    clean[spoiled] = 1.0
    want, wl, ob, lb = ref.attend(clean, k, v, ks, vs, table, lens, rows, causal, 1 / math.sqrt(dim))
    nan = spoiled & ~torch.isinf(wl)      # lse of -inf: the row sees nothing, or is not in use
    want[nan], wl[nan] = math.nan, math.nan
    compare(out, lse, want, wl, ob, lb)
    return out, lse, want, c, q


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("R,heads,copies", [(3, 2, 1), (70, 2, 20), (300, 8, 5)])      # the kernel for few rows, twice that for prompts
def test_every_score_is_minus_infinity(built_lib, cuda, dtype, dim, R, heads, copies):
    """An infinity of q on a column of K that has one sign: every score that the row sees is -inf (or +inf)."""
    lens, rows = [0, 1, 40, 200, 0, 33] * copies, [R, R, R - 1, R, 0, R] * copies

    def spoil(q, k, table):
        at = torch.zeros(q.shape[:3], dtype=torch.bool, device="cuda")
        k[..., 5] = k[..., 5].float().abs().clamp(min=1.0).to(k.dtype)
        q[0, 0, :, 5], q[1, R - 1, 0, 5], q[2, 1, 1, 5], q[3, R // 2, 0, 5], q[4, 0, 0, 5] = -math.inf, -math.inf, -math.inf, math.inf, -math.inf
        at[0, 0], at[1, R - 1, 0], at[2, 1, 1], at[3, R // 2, 0], at[4, 0, 0] = True, True, True, True, True
        return at
    attend(dtype, dim, heads, 1 if heads == 8 else 2, R, lens, rows, True, spoil)


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("R,copies", [(2, 1), (130, 16)])
def test_not_causal_mixed_signs_and_rows_that_see_nothing(built_lib, cuda, dtype, R, copies):
    lens = [0, 5, 300] * copies

    def spoil(q, k, table):
        at = torch.zeros(q.shape[:3], dtype=torch.bool, device="cuda")
        for b, i, h, d in ((0, 0, 0, 3), (1, 1, 2, 63), (2, 0, 3, 0), (2, R - 1, 1, 17)):
            q[b, i, h, d] = -math.inf if d % 2 else math.inf
            at[b, i, h] = True
        q[2, R - 1, 1, 18] = math.inf
        return at
    out, lse = attend(dtype, 64, 4, 2, R, lens, [R] * len(lens), False, spoil)[:2]
    assert bool((out[0] == 0).all()) and bool((lse[0] == -math.inf).all())


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_one_long_sequence_split_over_blocks(built_lib, cuda, dtype):
    def spoil(q, k, table):
        at = torch.zeros(q.shape[:3], dtype=torch.bool, device="cuda")
        k[..., 9] = (-k[..., 9].float().abs().clamp(min=1.0)).to(k.dtype)
        q[0, 1, 0, 9] = math.inf
        at[0, 1, 0] = True
        return at
    out, lse, want, c, q = attend(dtype, 64, 2, 1, 3, [20011], [3], True, spoil)
    again = c.attend(q, i32([20011]))
    assert same_bits(out, again[0]) and same_bits(lse, again[1])
