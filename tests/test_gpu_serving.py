"""The operators over a paged cache against plain 64-bit implementations."""
import math

import numpy as np
import pytest
import torch

import serving_ref as ref
from paper_2608_12703_gb300 import asrspec as A

pytestmark = pytest.mark.gpu

DT = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
LENS = [0, 1, 15, 16, 17, 31, 32, 33, 63, 100, 257, 700]


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def i32(x):
    return torch.tensor(list(x), dtype=torch.int32, device="cuda")


def pool(g, dtype, kv_heads, dim, page, need, layout="head"):
    """Pages scattered over a pool; unused slots hold NaN."""
    per = max(1, max(-(-n // page) for n in need))
    total = sum(-(-n // page) for n in need) + 2
    shape = (total, kv_heads, page, dim) if layout == "head" else (total, page, kv_heads, dim)
    k = torch.full(shape, math.nan, dtype=dtype, device="cuda")
    v = torch.full(shape, math.nan, dtype=dtype, device="cuda")
    if layout != "head":
        k, v = k.transpose(1, 2), v.transpose(1, 2)
    order = torch.randperm(total, generator=g, device="cuda").tolist()
    table, at = [], 0
    for n in need:
        p = -(-n // page)
        table.append(order[at:at + p] + [order[-1]] * (per - p))
        at += p
    table = torch.tensor(table, dtype=torch.int32, device="cuda")
    return k, v, table


def fill(g, pages, table, lens):
    page = pages.shape[2]
    for b, n in enumerate(lens):
        for j in range(-(-n // page)):
            m = min(page, n - j * page)
            pages[int(table[b, j]), :, :m] = torch.randn((pages.shape[1], m, pages.shape[3]), generator=g, device="cuda").to(pages.dtype)


def same_bits(a, b):
    return torch.equal(a.contiguous().view(torch.int16 if a.element_size() == 2 else torch.int32),
                       b.contiguous().view(torch.int16 if b.element_size() == 2 else torch.int32))


def check_attend(g, dtype, dim, heads, kv_heads, page, R, lens, rows, causal=True, append=True, layout="head", fused=True,
                 scale=None, spoil=None):
    from paper_2608_12703_gb300 import serving
    B = len(lens)
    need = [n + (R if causal else 0) for n in lens]
    k, v, table = pool(g, dtype, kv_heads, dim, page, need, layout)
    fill(g, k, table, lens)
    fill(g, v, table, lens)
    if fused:
        qkv = torch.randn((B, R, heads + 2 * kv_heads, dim), generator=g, device="cuda").to(dtype)
        q, kn, vn = qkv[:, :, :heads], qkv[:, :, heads:heads + kv_heads], qkv[:, :, heads + kv_heads:]
    else:   # heads outermost
        q = torch.randn((B, heads, R, dim), generator=g, device="cuda").to(dtype).transpose(1, 2)
        kn = torch.randn((B, kv_heads, R, dim), generator=g, device="cuda").to(dtype).transpose(1, 2)
        vn = torch.randn((B, kv_heads, R, dim), generator=g, device="cuda").to(dtype).transpose(1, 2)
    if spoil is not None:
        spoil(kn, vn)
    if not causal:
        append = False
    if not append:
        kr, vr = k.clone(), v.clone()
        if causal:
            for b in range(B):
                for i in range(rows[b]):
                    at = lens[b] + i
                    k[int(table[b, at // page]), :, at % page] = kn[b, i]
                    v[int(table[b, at // page]), :, at % page] = vn[b, i]
        kn = vn = None
    kr, vr = k.clone(), v.clone()
    c = serving.PagedCache(k, v, table)
    sc = 1 / math.sqrt(dim) if scale is None else scale
    out, lse = c.attend(q, i32(lens), k_new=kn, v_new=vn, rows=i32(rows), causal=causal, scale=scale)
    assert c.status() == 0
    want, wl, ob, lb = ref.attend(q, kr, vr, table, lens, rows, kn, vn, causal, sc)
    assert same_bits(k, kr) and same_bits(v, vr)
    fin = torch.isfinite(want)
    assert torch.equal(torch.isfinite(out.double()), fin)
    assert bool(((out.double() - want).abs()[fin] <= ob[fin]).all()), ((out.double() - want).abs() / ob)[fin].max()
    empty, none = torch.isinf(wl), torch.isnan(wl)      # rows that see no slot, and rows that see a NaN
    assert bool((lse[empty] == -math.inf).all()) and torch.equal(torch.isnan(lse), none)
    sure = ~(empty | none)
    assert bool(((lse.double() - wl).abs()[sure] <= lb[sure]).all())
    again, lse2 = c.attend(q, i32(lens), k_new=kn, v_new=vn, rows=i32(rows), causal=causal, scale=scale)
    assert same_bits(out, again) and same_bits(lse, lse2)   # the order of the work does not show


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("dim,heads,kv_heads,page,R", [
    (64, 3, 3, 16, 1), (64, 4, 4, 48, 9), (64, 8, 2, 32, 7), (128, 4, 1, 16, 1), (128, 6, 2, 64, 5), (64, 16, 1, 16, 5)])
def test_attend_matches_plain(built_lib, cuda, dtype, dim, heads, kv_heads, page, R):
    g = gen(dim + heads * 3 + page + R)
    rows = [R if i % 3 else (i * 5) % (R + 1) for i in range(len(LENS))]
    check_attend(g, DT[dtype], dim, heads, kv_heads, page, R, LENS, rows)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("layout,fused", [("slot", True), ("head", False), ("slot", False)])
def test_attend_strides(built_lib, cuda, dtype, layout, fused):
    check_attend(gen(5), DT[dtype], 64, 6, 3, 16, 4, [0, 5, 40, 130], [4, 0, 3, 4], layout=layout, fused=fused)


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("dim", [64, 128])
def test_attend_not_causal_and_block_in_pages(built_lib, cuda, dtype, dim):
    check_attend(gen(6), DT[dtype], dim, 4, 2, 32, 3, [0, 1, 33, 300], [3, 3, 2, 0], causal=False)
    check_attend(gen(7), DT[dtype], dim, 4, 2, 32, 3, [0, 1, 33, 300], [3, 3, 2, 0], append=False)


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
def test_attend_scales(built_lib, cuda, dtype):
    check_attend(gen(8), DT[dtype], 64, 2, 2, 16, 2, [50, 120], [2, 1], scale=1e-3)
    check_attend(gen(9), DT[dtype], 64, 2, 2, 16, 2, [50, 120], [2, 1], scale=2.0)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_attend_one_long_sequence(built_lib, cuda, dtype):
    """Every head split over many warps and joined."""
    check_attend(gen(10), DT[dtype], 64, 2, 1, 16, 3, [20011], [3])


def test_attend_many_sequences(built_lib, cuda):
    lens = [(i * 37) % 90 for i in range(70)]
    check_attend(gen(11), DT["bf16"], 64, 2, 2, 16, 2, lens, [i % 3 for i in range(70)])


@pytest.mark.parametrize("dtype,dim,R", [("bf16", 64, 2), ("bf16", 64, 11), ("fp16", 128, 9), ("fp32", 64, 3)])
def test_attend_long_among_many_short(built_lib, cuda, dtype, dim, R):
    """More sequences than are ranked by length: equal runs of steps, one item spread over many warps and blocks."""
    lens = [3] * 150 + [9001] + [5] * 140
    check_attend(gen(16), DT[dtype], dim, 1, 1, 16, R, lens, [R] * 150 + [R] + [1] * 140)


def test_attend_most_sequences(built_lib, cuda):
    check_attend(gen(17), DT["bf16"], 64, 1, 1, 16, 1, [(i * 5) % 40 for i in range(1024)], [i % 2 for i in range(1024)])


@pytest.mark.parametrize("dtype,dim,heads,kv_heads", [("bf16", 64, 6, 3), ("bf16", 128, 4, 2), ("fp32", 128, 2, 2)])
def test_attend_few_long_items(built_lib, cuda, dtype, dim, heads, kv_heads):
    """Fewer items than blocks: each shared by several."""
    check_attend(gen(18), DT[dtype], dim, heads, kv_heads, 48, 5, [6000, 1, 4100], [5, 5, 2])


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("dim", [64, 128])
def test_attend_hidden_rows_do_not_leak(built_lib, cuda, dtype, dim):
    """Infinities and NaN in a later draft's K and V reach only the rows that see it; slots past the block hold NaN."""
    def spoil(kn, vn):
        vn[0, 2, 0, 3] = math.inf
        vn[1, 3, 0, :] = math.nan
        vn[2, 1, 1, dim - 1] = -math.inf
        kn[3, 3, 0, 0] = math.nan
        vn[4, 3, 1, 8] = math.inf
    check_attend(gen(12), DT[dtype], dim, 4, 2, 16, 4, [0, 14, 29, 61, 47], [4, 4, 4, 4, 3], spoil=spoil)


def test_attend_pages_past_32_bit_offsets(built_lib, cuda):
    """Page ids whose byte offsets pass 2^32 and element offsets 2^31."""
    from paper_2608_12703_gb300 import serving
    g = gen(13)
    K, D, page = 20, 64, 16
    n_pages = (1 << 32) // (K * D * page * 2) + 4 + (1 << 31) // (K * D * page)
    k = torch.empty((n_pages, K, page, D), dtype=torch.bfloat16, device="cuda")
    v = torch.empty_like(k)
    table = torch.tensor([[n_pages - 1, 3, n_pages - 2]], dtype=torch.int32, device="cuda")
    fill(g, k, table, [37])
    fill(g, v, table, [37])
    q, kn, vn = (torch.randn((1, 2, K, D), generator=g, device="cuda").bfloat16() for _ in range(3))
    out, lse = serving.PagedCache(k, v, table).attend(q, i32([37]), k_new=kn, v_new=vn)
    ids = table[0].long()
    small = torch.tensor([[0, 1, 2]], dtype=torch.int32)
    want, wl, ob, lb = ref.attend(q, k[ids].clone(), v[ids].clone(), small, [37], [2], kn, vn, True, 0.125)
    assert bool(((out.double() - want).abs() <= ob).all()) and bool(((lse.double() - wl).abs() <= lb).all())
    assert torch.equal(k[n_pages - 2][:, 5:7].transpose(0, 1), kn[0])


def test_attend_data_errors(built_lib, cuda):
    """Bad lengths and rows leave the sequence's rows zero, and they and a bad page id leave its pages alone; the other
    sequences are computed."""
    from paper_2608_12703_gb300 import serving
    g = gen(14)
    k, v, table = pool(g, torch.bfloat16, 2, 64, 16, [32] * 4)
    fill(g, k, table, [32] * 4)
    fill(g, v, table, [32] * 4)
    q, kn, vn = (torch.randn((4, 2, 2, 64), generator=g, device="cuda").bfloat16() for _ in range(3))
    ok, _ = serving.PagedCache(k.clone(), v.clone(), table).attend(q, i32([20] * 4), k_new=kn, v_new=vn)
    for lens, rows, bit in (([20, 31, 20, 20], [2, 2, 2, 2], A.ST_CAPACITY), ([20, -1, 20, 20], [2, 2, 2, 2], A.ST_CAPACITY),
                            ([20, 20, 20, 20], [2, 3, 2, 2], A.ST_BAD_LENS), ([20, 20, 20, 20], [2, -1, 2, 2], A.ST_BAD_LENS),
                            (None, None, A.ST_BOUNDS)):
        t = table.clone()
        if lens is None:
            lens, rows = [20] * 4, [2] * 4
            t[1, 1] = k.shape[0]
        kk, vv = k.clone(), v.clone()
        c = serving.PagedCache(kk, vv, t)
        out, lse = c.attend(q, i32(lens), k_new=kn, v_new=vn, rows=i32(rows))
        assert c.status() == bit
        assert c.status() == 0
        if bit != A.ST_BOUNDS:
            assert bool((out[1] == 0).all()) and bool((lse[1] == -math.inf).all())
        for b in (0, 2, 3):
            assert same_bits(out[b], ok[b])
            at = t[b, 1].long()          # slots 20 and 21
            assert same_bits(kk[at][:, 4:6], kn[b].transpose(0, 1)) and same_bits(vv[at][:, 4:6], vn[b].transpose(0, 1))
            kk[at], vv[at] = k[at], v[at]
        assert same_bits(kk, k) and same_bits(vv, v)   # nothing else was written


def test_attend_side_stream_and_graph(built_lib, cuda):
    from paper_2608_12703_gb300 import serving
    g = gen(15)
    k, v, table = pool(g, torch.bfloat16, 4, 64, 16, [320, 100])
    fill(g, k, table, [300, 90])
    fill(g, v, table, [300, 90])
    q, kn, vn = (torch.randn((2, 3, 4, 64), generator=g, device="cuda").bfloat16() for _ in range(3))
    n = i32([300, 90])
    c = serving.PagedCache(k, v, table)
    want, wl = c.attend(q, n, k_new=kn, v_new=vn)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        out, lse = c.attend(q, n, k_new=kn, v_new=vn)
    side.synchronize()
    assert same_bits(out, want) and same_bits(lse, wl)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out, lse = c.attend(q, n, k_new=kn, v_new=vn)
    out.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert same_bits(out, want) and same_bits(lse, wl)


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("dim,heads,kv_heads,page,R,causal", [
    (64, 3, 3, 16, 1, True), (64, 4, 4, 48, 9, True), (64, 16, 2, 32, 5, True), (128, 4, 1, 16, 1, True), (128, 6, 2, 64, 5, False)])
def test_weigh_matches_plain(built_lib, cuda, dtype, dim, heads, kv_heads, page, R, causal):
    from paper_2608_12703_gb300 import serving
    g = gen(20 + dim + heads + R)
    lens = LENS
    B = len(lens)
    k, v, table = pool(g, DT[dtype], kv_heads, dim, page, [n + R for n in lens])
    fill(g, k, table, [n + R for n in lens])
    v.zero_()
    q = torch.randn((B, R, heads, dim), generator=g, device="cuda").to(DT[dtype])
    rows = [R if i % 3 else (i * 5) % (R + 1) for i in range(B)]
    c = serving.PagedCache(k, v, table)
    _, lse = c.attend(q, i32(lens), causal=causal)
    lse[3, 0, 0] = -math.inf
    cap = max(lens) + R + 3
    score = torch.rand((B, kv_heads, cap), generator=g, device="cuda") * 3
    for b, n in enumerate(lens):
        score[b, :, n:] = math.nan      # stale entries of the slots that the block takes
    pos = torch.full((B, kv_heads, cap), -7, dtype=torch.int32, device="cuda")
    first = i32([10 * n + 1 for n in lens])
    out = torch.full_like(score, -5.0)
    got = c.weigh(q, lse, i32(lens), score, rows=i32(rows), causal=causal, out=out, pos=pos, first_pos=first)
    assert got is out and c.status() == 0
    want, bound = ref.weigh(q, lse, k, table, lens, rows, score, causal, 1 / math.sqrt(dim))
    live = ~torch.isnan(want)
    assert bool((out[~live] == -5.0).all())
    assert bool(((out.double() - want).abs()[live] <= bound[live]).all())
    for b, n in enumerate(lens):
        for i in range(cap - n):
            new = causal and i < rows[b]
            assert bool((pos[b, :, n + i] == (10 * n + 1 + i if new else -7)).all())
    inplace = score.clone()
    c.weigh(q, lse, i32(lens), inplace, rows=i32(rows), causal=causal)
    assert torch.equal(inplace[live], out[live])
    fresh = c.weigh(q, lse, i32(lens), None, rows=i32(rows), causal=causal, out=torch.full_like(score, -5.0))
    want0, bound0 = ref.weigh(q, lse, k, table, lens, rows, torch.zeros_like(score), causal, 1 / math.sqrt(dim))
    assert bool(((fresh.double() - want0).abs()[live] <= bound0[live]).all())


def test_weights_of_a_row_sum_to_one(built_lib, cuda):
    from paper_2608_12703_gb300 import serving
    g = gen(30)
    k, v, table = pool(g, torch.bfloat16, 4, 64, 16, [1001])
    fill(g, k, table, [1000])
    fill(g, v, table, [1000])
    q, kn, vn = (torch.randn((1, 1, 4, 64), generator=g, device="cuda").bfloat16() for _ in range(3))
    c = serving.PagedCache(k, v, table)
    _, lse = c.attend(q, i32([1000]), k_new=kn, v_new=vn)
    s = c.weigh(q, lse, i32([1000]), None, out=torch.zeros((1, 4, 1001), device="cuda"))
    # scores of at most 9 or so: lse and weights each within (64 + 8) 2^-22 * 9 and 2^-18 of exact
    assert bool(((s.double().sum(2) - 1).abs() < 4e-4).all())


def check_evict(g, dtype, kv_heads, dim, page, lens, budget, recent, first, score, pos, seen, inplace=False):
    from paper_2608_12703_gb300 import serving
    B = len(lens)
    k, v, table = pool(g, dtype, kv_heads, dim, page, lens)
    fill(g, k, table, lens)
    fill(g, v, table, lens)
    k0, v0 = k.clone(), v.clone()
    c = serving.PagedCache(k, v, table)
    s0, p0 = score.clone(), pos.clone()
    if inplace:
        lens_d = i32(lens)
        out = c.evict(lens_d, score, pos, i32(seen), budget=budget, recent=recent, first=first, lens_out=lens_d)
        assert out[0] is lens_d and out[1] is score and out[2] is pos
    else:
        cap = max(1, min(budget, max(lens)))
        out = c.evict(i32(lens), score, pos, i32(seen), budget=budget, recent=recent, first=first,
                      score_out=torch.zeros((B, kv_heads, cap), device="cuda"),
                      pos_out=torch.zeros((B, kv_heads, cap), dtype=torch.int32, device="cuda"))
        assert same_bits(score, s0) and torch.equal(pos, p0)
    assert c.status() == 0
    plan = ref.evict(lens, s0.cpu(), p0.cpu(), seen, budget, recent, first)
    assert out[0].tolist() == [min(n, budget) for n in lens]
    for b, n in enumerate(lens):
        m = min(n, budget)
        for h in range(kv_heads):
            order = torch.tensor(plan[b][h], dtype=torch.long, device="cuda")
            assert len(plan[b][h]) == m
            assert same_bits(out[1][b, h, :m], s0[b, h][order]) and torch.equal(out[2][b, h, :m], p0[b, h][order])
        for new, old in ((k, k0), (v, v0)):
            a, o = ref.slots(new, table[b], n), ref.slots(old, table[b], n)
            for h in range(kv_heads):
                order = torch.tensor(plan[b][h] + list(range(m, n)), dtype=torch.long, device="cuda")
                assert torch.equal(a[:, h], o[order, h])


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("dim,page", [(64, 16), (128, 48)])
@pytest.mark.parametrize("inplace", [False, True])
def test_evict_matches_plain(built_lib, cuda, dtype, dim, page, inplace):
    g = gen(40)
    lens, K = [0, 1, 39, 40, 41, 80, 555, 700], 3
    score = torch.rand((len(lens), K, 700), generator=g, device="cuda")
    score = torch.where(score < 0.6, torch.round(score * 8) / 8, score)     # equal scores across the cut
    pos = torch.stack([torch.randperm(900, generator=g, device="cuda")[:700] for _ in range(len(lens) * K)]).to(torch.int32)
    check_evict(g, DT[dtype], K, dim, page, lens, 40, 10, 4, score, pos.view(len(lens), K, 700), [900] * len(lens), inplace)


@pytest.mark.parametrize("case", ["equal", "protected", "odd", "sorted", "one", "half"])
def test_evict_edges(built_lib, cuda, case):
    """All scores equal; more protected slots than the budget; infinities, NaN and negative scores; best slots all past the
    budget; a budget of one; two equal halves."""
    g = gen(41)
    n, K = 1300, 2
    budget, recent, first = 500, 0, 0
    score = torch.rand((2, K, n), generator=g, device="cuda")
    pos = torch.arange(n, device="cuda", dtype=torch.int32).repeat(2, K, 1).contiguous()
    if case == "equal":
        score.fill_(0.25)
    elif case == "protected":
        recent, first = 700, 40
    elif case == "odd":
        score[:, :, ::3] = math.nan
        score[:, :, 1::7] = math.inf
        score[:, :, 2::5] = -1.0
        score[:, :, 3::11] = -math.inf
        score[:, :, 4::13] = -0.0
        score[:, :, 5::13] = 0.0
        budget = 1250
    elif case == "sorted":
        score = torch.arange(n, device="cuda", dtype=torch.float32).repeat(2, K, 1).contiguous()
    elif case == "one":
        budget = 1
    elif case == "half":
        score[:, :, :650], score[:, :, 650:] = 1.0, 2.0
        budget = 650
    check_evict(g, torch.bfloat16, K, 64, 32, [n, n - 7], budget, recent, first, score, pos, [n, n])


def test_evict_long(built_lib, cuda):
    g = gen(42)
    lens = [20001, 17000]
    score = torch.empty((2, 2, 20001), device="cuda").log_normal_(generator=g)
    pos = torch.arange(20001, device="cuda", dtype=torch.int32).repeat(2, 2, 1).contiguous()
    check_evict(g, torch.bfloat16, 2, 64, 64, lens, 9000, 64, 4, score, pos, lens)


def test_evict_data_errors(built_lib, cuda):
    from paper_2608_12703_gb300 import serving
    g = gen(43)
    k, v, table = pool(g, torch.bfloat16, 2, 64, 16, [64, 64])
    fill(g, k, table, [64, 64])
    fill(g, v, table, [64, 64])
    k0 = k.clone()
    score = torch.rand((2, 2, 64), generator=g, device="cuda")
    pos = torch.arange(64, device="cuda", dtype=torch.int32).repeat(2, 2, 1).contiguous()
    c = serving.PagedCache(k, v, table)
    n, _, _ = c.evict(i32([65, 64]), score, pos, i32([64, 64]), budget=32)
    assert c.status() == A.ST_CAPACITY and n.tolist() == [65, 32]
    assert torch.equal(k[table[0].long()], k0[table[0].long()])


def make_accept(seed, dtype, B, k, V, with_q, temperature, shift=0):
    g = gen(seed)

    def logits(rows):
        store = torch.empty(B * rows * V + 8, dtype=dtype, device="cuda")
        x = store[shift:shift + B * rows * V].view(B, rows, V)
        x.copy_((torch.randn((B, rows, V), generator=g, device="cuda") * 2.5).to(dtype))
        return x
    target = logits(k + 1)
    dl = None
    if with_q:
        dl = logits(k) if k else torch.empty((B, 0, V), dtype=dtype, device="cuda")
        if k:
            dl.copy_((target[:, :k].float() + 0.7 * torch.randn((B, k, V), generator=g, device="cuda")).to(dtype))
    draft = (dl if with_q else target[:, :k]).float()
    draft = (draft / temperature - torch.empty((B, k, V), device="cuda").exponential_(generator=g).log()).argmax(2).to(torch.int32) \
        if k else torch.zeros((B, 0), dtype=torch.int32, device="cuda")
    lens = i32([k if i % 4 else (i * 3) % (k + 2) - 1 for i in range(B)])
    u = torch.rand((B, k), generator=g, device="cuda")
    race = torch.empty((B, V), device="cuda").exponential_(generator=g).clamp_(min=1e-30)
    return target, draft, lens, u, race, dl


def check_accept(target, draft, lens, u, race, dl, temperature):
    from paper_2608_12703_gb300 import serving
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    got = serving.accept_sampled(target, draft, lens, u, race, draft_logits=dl, temperature=temperature, status=status)
    acc, tok, step, prob, margin = ref.accept(target.double().cpu().numpy(), draft.cpu().numpy(), lens.cpu().numpy(),
                                              u.double().cpu().numpy(), race.cpu().numpy(),
                                              None if dl is None else dl.double().cpu().numpy(), temperature)
    # A logit's distance to the maximum is rounded at 2^-24 and scaled by log2(e) / T: p is off by at most
    # 2^-21 (1 + spread / T) in relation; decisions closer than that are not fixed by the definition.
    x = target.float()
    spread = float(x[x.abs() < 1e4].abs().max()) * 2    # masked and infinite logits have weights of exactly 0 or 1
    tol = 2.0 ** -20 * (1 + spread / temperature)
    sure = margin > 4 * tol
    assert sure.mean() > 0.9
    a, t, s, p = (x.cpu().numpy() for x in got)
    assert np.array_equal(a[sure], acc[sure]) and np.array_equal(t[sure], tok[sure]) and np.array_equal(s[sure], step[sure])
    assert np.all(np.abs(p - prob) <= 4 * tol * prob + 1e-30)
    assert int(status) == 0
    return got


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("with_q", [True, False])
@pytest.mark.parametrize("B,k,V,temperature,shift", [
    (5, 4, 51866, 1.0, 0), (9, 3, 51865, 0.7, 1), (3, 0, 1001, 1.0, 3), (40, 7, 17, 1.3, 5), (6, 31, 333, 0.2, 2), (4, 2, 1, 1.0, 1)])
def test_accept_matches_plain(built_lib, cuda, dtype, with_q, B, k, V, temperature, shift):
    x = make_accept(50 + k + B, DT[dtype], B, k, V, with_q, temperature, shift)
    check_accept(*x, temperature)


def test_accept_strided_rows(built_lib, cuda):
    """Logits that are slices of padded rows, race rows of a wider buffer, one set of target rows shared by all."""
    t, d, n, u, r, q = make_accept(60, torch.float32, 6, 3, 1003, True, 1.0)
    wide = torch.full((6, 4, 1100), 1e4, device="cuda")
    wide[:, :, 5:1008] = t
    rw = torch.full((6, 1100), 1e-30, device="cuda")
    rw[:, 7:1010] = r
    want = check_accept(t, d, n, u, r, q, 1.0)
    got = check_accept(wide[:, :, 5:1008], d, n, u, rw[:, 7:1010], q, 1.0)
    for a, b in zip(want[:3], got[:3]):
        assert torch.equal(a, b)
    check_accept(t[:1].expand(6, 4, 1003), d, n, u, r, q, 1.0)


def test_accept_masked_logits(built_lib, cuda):
    """Masked tokens (-inf, NaN), the type's lowest value as a mask, a row with nothing left, +inf."""
    t, d, n, u, r, q = make_accept(61, torch.float32, 8, 3, 500, True, 1.0)
    n = i32([3] * 8)
    t[:, :, ::2] = -math.inf
    t[:, :, 1::4] = math.nan
    t[1, :, 3::8] = -3.4028234e38
    t[2, 0] = -math.inf               # the first row has no token left
    t[3, :] = -math.inf
    t[4, 1] = -3.4028234e38           # every logit the lowest value: uniform
    t[5, 0, 7] = math.inf
    q[6, 0] = -math.inf               # the draft's row has nothing: q = 0
    d[:, 0] = 7                       # an unmasked token
    got = check_accept(t, d, n, u, r, q, 1.0)
    assert int(got[1][2]) == -1 and int(got[2][2]) == 0 and int(got[0][2]) == 0
    assert int(got[1][3]) == -1
    assert int(got[0][5]) >= 1


def test_accept_draft_equal_to_target(built_lib, cuda):
    """p = q accepts every draft for every u < 1."""
    t, d, n, u, r, _ = make_accept(62, torch.bfloat16, 16, 5, 3000, True, 0.9)
    from paper_2608_12703_gb300 import serving
    u.fill_(1.0 - 2.0 ** -24)
    n = i32([5] * 16)
    acc, tok, step, prob = serving.accept_sampled(t, d, n, u, r, draft_logits=t[:, :5].contiguous(), temperature=0.9)
    assert bool((acc == 5).all()) and bool((step == 6).all()) and bool((prob == 1).all())


def test_accept_tokens_follow_the_target(built_lib, cuda):
    """Over many utterances that share their logits the first emitted token has the target's distribution, whatever the
    draft's: chi-square with 7 degrees of freedom below 35 (chance 1e-5)."""
    from paper_2608_12703_gb300 import serving
    g = gen(63)
    N, V = 60000, 8
    t = (torch.randn((1, 2, V), generator=g, device="cuda")).expand(N, 2, V)
    q = (torch.randn((1, 1, V), generator=g, device="cuda")).expand(N, 1, V)
    race = lambda: torch.empty((N, V), device="cuda").exponential_(generator=g).clamp_(min=1e-30)
    for dl in (q, None):
        d = (q[:, 0] - race().log()).argmax(1).to(torch.int32)[:, None].contiguous()
        acc, tok, _, _ = serving.accept_sampled(t, d, None, torch.rand((N, 1), generator=g, device="cuda"), race(),
                                                draft_logits=dl)
        first = torch.where(acc == 1, d[:, 0], tok)
        p = torch.softmax(t[0, 0].double(), 0).cpu()
        have = torch.bincount(first.long(), minlength=V).double().cpu()
        assert float(((have - N * p) ** 2 / (N * p)).sum()) < 35


def test_accept_data_errors(built_lib, cuda):
    from paper_2608_12703_gb300 import serving
    t, d, n, u, r, q = make_accept(64, torch.float32, 4, 3, 100, True, 1.0)
    n = i32([3] * 4)
    good = serving.accept_sampled(t, d, n, u, r, draft_logits=q)
    for bad, bit in (("token", A.ST_BAD_TOKEN), ("low", A.ST_BAD_TOKEN), ("lens", A.ST_BAD_LENS), ("neg", A.ST_BAD_LENS)):
        dd, nn = d.clone(), n.clone()
        if bad in ("token", "low"):
            dd[2, 1] = 100 if bad == "token" else -1
        else:
            nn[2] = 4 if bad == "lens" else -2
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        got = serving.accept_sampled(t, dd, nn, u, r, draft_logits=q, status=status)
        assert int(status) == bit
        assert [int(x[2]) for x in got[:3]] == [0, -1, 0] and bool((got[3][2] == 0).all())
        for b in (0, 1, 3):
            assert all(torch.equal(x[b], y[b]) for x, y in zip(good, got))


def test_refusals(built_lib, cuda):
    from paper_2608_12703_gb300 import serving
    z = lambda *s, dt=torch.bfloat16: torch.zeros(s, dtype=dt, device="cuda")
    k, v, t = z(4, 2, 16, 64), z(4, 2, 16, 64), z(2, 2, dt=torch.int32)
    n = z(2, dt=torch.int32)

    def refused(f):
        with pytest.raises(A.AsrSpecError, match="ASR_E_INVAL"):
            f()
    P = serving.PagedCache
    for args in ((k.cpu(), v, t), (k, v.float(), t), (k, v, t.long()), (z(4, 2, 15, 64), z(4, 2, 15, 64), t),
                 (z(4, 2, 16, 96), z(4, 2, 16, 96), t), (k, z(4, 2, 16, 128)[..., :64], t), (k.double(), v.double(), t)):
        refused(lambda: P(*args))
    c = P(k, v, t)
    q = z(2, 3, 4, 64)
    for kw in (dict(q=z(2, 3, 3, 64)), dict(q=z(1, 3, 4, 64)), dict(q=q.half()), dict(q=q.cpu()), dict(kv_len=n.long()),
               dict(kv_len=n[:1]), dict(rows=z(3, dt=torch.int32)), dict(k_new=z(2, 3, 2, 64)),
               dict(k_new=z(2, 3, 2, 64), v_new=z(2, 3, 2, 64), causal=False), dict(k_new=z(2, 3, 4, 64), v_new=z(2, 3, 4, 64)),
               dict(scale=0.0), dict(scale=float("nan")), dict(q=z(2, 3, 4, 65)[..., 1:]), dict(out=z(2, 3, 4, 32)),
               dict(lse=z(2, 3, 4))):
        kw = {"q": q, "kv_len": n, **kw}
        refused(lambda: c.attend(kw.pop("q"), kw.pop("kv_len"), **kw))
    lse, s, p = z(2, 3, 4, dt=torch.float32), z(2, 2, 32, dt=torch.float32), z(2, 2, 32, dt=torch.int32)
    refused(lambda: c.weigh(q, lse, n, None))
    refused(lambda: c.weigh(q, lse, n, s.half()))
    refused(lambda: c.weigh(q, lse, n, s, pos=p))
    refused(lambda: c.weigh(q, lse[:, :2], n, s))
    refused(lambda: c.evict(n, s, p, n, budget=0))
    refused(lambda: c.evict(n, s, p.float(), n, budget=4))
    refused(lambda: c.evict(n, s, p, n, budget=4, score_out=z(2, 2, 8, dt=torch.float32)))
    x = (z(2, 3, 9, dt=torch.float32), z(2, 2, dt=torch.int32), n, z(2, 2, dt=torch.float32), z(2, 9, dt=torch.float32))
    S = serving.accept_sampled
    refused(lambda: S(x[0].cpu(), *x[1:]))
    refused(lambda: S(x[0], x[1].long(), *x[2:]))
    refused(lambda: S(*x, temperature=0.0))
    refused(lambda: S(*x, draft_logits=z(2, 2, 9)))
    refused(lambda: S(*x[:4], x[4][:, :8]))
    refused(lambda: S(z(2, 34, 9, dt=torch.float32), *x[1:]))
    assert c.status() == 0


def test_evict_longest_heads(built_lib, cuda):
    """More slots a block than one of ordinary size keeps ranks of; and, of the same lengths, more than any keeps."""
    g = gen(44)
    for n, budget in ((70001, 30000), (330003, 329000)):
        score = torch.empty((1, 1, n), device="cuda").log_normal_(generator=g)
        pos = torch.arange(n, device="cuda", dtype=torch.int32).view(1, 1, n).contiguous()
        check_evict(g, torch.bfloat16, 1, 64, 1024, [n], budget, 64, 4, score, pos, [n])
