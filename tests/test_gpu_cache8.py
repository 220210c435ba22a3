"""Attention over an 8-bit paged cache, and the append to it, against plain 64-bit implementations."""
import math

import pytest
import torch

import cache8_ref as ref
from paper_2608_12703_gb300 import asrspec as A

pytestmark = pytest.mark.gpu

DT = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
LENS = [0, 1, 15, 16, 17, 31, 32, 33, 63, 65, 100, 257, 700]


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def i32(x):
    return torch.tensor(list(x), dtype=torch.int32, device="cuda")


def randn(g, *shape):
    return torch.randn(shape, generator=g, device="cuda")


def pool(g, kv_heads, dim, page, need, layout="head"):
    """Pages scattered over a pool; every slot a NaN, every scale one too."""
    per = max(1, max(-(-n // page) for n in need))
    total = sum(-(-n // page) for n in need) + 2
    shape = (total, kv_heads, page, dim) if layout == "head" else (total, page, kv_heads, dim)
    k, v = (torch.full(shape, 0x7f, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn) for _ in range(2))
    if layout != "head":
        k, v = k.transpose(1, 2), v.transpose(1, 2)
    ks, vs = (torch.full((total, kv_heads, page // 16), math.nan, device="cuda") for _ in range(2))
    order = torch.randperm(total, generator=g, device="cuda").tolist()
    table, at = [], 0
    for n in need:
        p = -(-n // page)
        table.append(order[at:at + p] + [order[-1]] * (per - p))
        at += p
    return k, v, ks, vs, i32(sum(table, [])).reshape(len(need), per)


def fill(g, pages, scales, table, lens, spread=2):
    """Codes over their type's whole range; scales of several powers of two."""
    page = pages.shape[2]
    for b, n in enumerate(lens):
        for j in range(-(-n // page)):
            pid, m = int(table[b, j]), min(page, n - j * page)
            x = (randn(g, pages.shape[1], m, pages.shape[3]) * 100).clamp(-448, 448)
            pages[pid, :, :m] = x.to(pages.dtype)
            used = -(-m // 16)
            e = torch.randint(-7 - spread, -6, (pages.shape[1], used), generator=g, device="cuda")
            scales[pid, :, :used] = torch.exp2(e.float())


def codes(x):
    return x.contiguous().view(torch.uint8)


def same_bits(a, b):
    return torch.equal(a.contiguous().view(torch.uint8), b.contiguous().view(torch.uint8))


def make_rows(g, B, R, heads, kv_heads, dim, dtype, fused):
    if fused:
        qkv = randn(g, B, R, heads + 2 * kv_heads, dim).to(dtype)
        return qkv[:, :, :heads], qkv[:, :, heads:heads + kv_heads], qkv[:, :, heads + kv_heads:]
    return [randn(g, B, h, R, dim).to(dtype).transpose(1, 2) for h in (heads, kv_heads, kv_heads)]


def compare(out, lse, want, wl, ob, lb):
    # a value from half a step beyond the type's largest on rounds to infinity; within the bound of that point it may or may not
    top = torch.finfo(out.dtype).max * (1 + torch.finfo(out.dtype).eps / 4)
    over, fin = want.abs() - ob >= top, want.abs() + ob < top
    assert bool((out[over].double() == want[over].sign() * math.inf).all())
    assert bool(torch.isfinite(out[fin]).all()) and torch.equal(torch.isnan(out), torch.isnan(want))
    assert bool(((out.double() - want).abs()[fin] <= ob[fin]).all()), ((out.double() - want).abs() / ob)[fin].max()
    empty, none = torch.isinf(wl), torch.isnan(wl)
    assert bool((lse[empty] == -math.inf).all()) and torch.equal(torch.isnan(lse), none)
    sure = ~(empty | none)
    assert bool(((lse.double() - wl).abs()[sure] <= lb[sure]).all()), ((lse.double() - wl).abs() / lb)[sure].max()


def check(g, dtype, dim, heads, kv_heads, page, R, lens, rows, causal=True, append=True, layout="head", fused=True, scale=None,
          spoil=None, spread=2):
    from paper_2608_12703_gb300 import serving
    B = len(lens)
    k, v, ks, vs, table = pool(g, kv_heads, dim, page, [n + (R if causal else 0) for n in lens], layout)
    fill(g, k, ks, table, lens, spread)
    fill(g, v, vs, table, lens, spread)
    q, kn, vn = make_rows(g, B, R, heads, kv_heads, dim, dtype, fused)
    if spoil is not None:
        spoil(q, kn, vn, v, vs, table)
    kr, vr, ksr, vsr = k.clone(), v.clone(), ks.clone(), vs.clone()
    if causal:
        ref.append(kr, ksr, table, lens, rows, kn)
        ref.append(vr, vsr, table, lens, rows, vn)
    c = serving.PagedCache8(k, v, ks, vs, table)
    if causal and not append:
        c.append(kn, vn, i32(lens), rows=i32(rows))
        kn = vn = None
    if not causal:
        kn = vn = None
    out, lse = c.attend(q, i32(lens), k_new=kn, v_new=vn, rows=i32(rows), causal=causal, scale=scale)
    assert c.status() == 0
    assert torch.equal(codes(k), codes(kr)) and torch.equal(codes(v), codes(vr))
    assert same_bits(ks, ksr) and same_bits(vs, vsr)
    compare(out, lse, *ref.attend(q, kr, vr, ksr, vsr, table, lens, rows, causal, 1 / math.sqrt(dim) if scale is None else scale))
    out2, lse2 = c.attend(q, i32(lens), k_new=kn, v_new=vn, rows=i32(rows), causal=causal, scale=scale)
    assert same_bits(out, out2) and same_bits(lse, lse2)   # the order of the work does not show, nor a second append
    assert torch.equal(codes(k), codes(kr)) and same_bits(ks, ksr)


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("dim,heads,kv_heads,page,R", [
    (64, 3, 3, 16, 1), (64, 4, 4, 48, 9), (64, 8, 2, 32, 7), (128, 4, 1, 16, 1), (128, 6, 2, 64, 5), (64, 16, 1, 16, 5),
    (64, 1, 1, 16, 33), (128, 8, 1, 32, 2)])
def test_attend_matches_plain(built_lib, cuda, dtype, dim, heads, kv_heads, page, R):
    rows = [R if i % 3 else (i * 5) % (R + 1) for i in range(len(LENS))]
    check(gen(dim + heads * 3 + page + R), DT[dtype], dim, heads, kv_heads, page, R, LENS, rows)


@pytest.mark.parametrize("layout,fused", [("slot", True), ("head", False), ("slot", False)])
def test_attend_strides(built_lib, cuda, layout, fused):
    check(gen(5), DT["bf16"], 64, 6, 3, 16, 4, [0, 5, 40, 130], [4, 0, 3, 4], layout=layout, fused=fused)
    check(gen(6), DT["fp16"], 128, 6, 3, 48, 4, [0, 5, 40, 130], [4, 0, 3, 4], layout=layout, fused=fused)


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("dim", [64, 128])
def test_attend_not_causal_and_append_apart(built_lib, cuda, dtype, dim):
    check(gen(6), DT[dtype], dim, 4, 2, 32, 3, [0, 1, 33, 300], [3, 3, 2, 0], causal=False)
    check(gen(7), DT[dtype], dim, 4, 2, 32, 3, [0, 1, 33, 300], [3, 3, 2, 0], append=False)


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("dim,heads,kv_heads,R", [(64, 3, 3, 130), (128, 4, 2, 70), (64, 8, 1, 40), (64, 2, 2, 300)])
@pytest.mark.parametrize("copies", [1, 8])
def test_attend_prompts(built_lib, cuda, dtype, dim, heads, kv_heads, R, copies):
    """Prompts, on their own and behind what is there already; not causal besides.  Few of them, and enough to fill the GPU."""
    lens, rows = [0, 7, 16, 130, 500] * copies, [R, R - 1, 17, R, 1] * copies
    check(gen(8), DT[dtype], dim, heads, kv_heads, 32, R, lens, rows)
    check(gen(9), DT[dtype], dim, heads, kv_heads, 16, R, lens, rows, causal=False, fused=False)


@pytest.mark.parametrize("dtype,dim,causal", [("bf16", 64, True), ("fp16", 64, False), ("bf16", 128, True), ("fp16", 128, False)])
def test_attend_many_prompts(built_lib, cuda, dtype, dim, causal):
    """Many prompts a block, of one row tile and of several, with sequences that sit out and that see nothing between them."""
    g, B, K = gen(dim), 40, 24
    R = 290
    rows = [(0, 70, R, 128, 200, 129, 256, 1, 257, 65)[i % 10] for i in range(B)]
    check(g, DT[dtype], dim, K, K, 16, R, [(i * 29) % 300 if i % 7 else 0 for i in range(B)], rows, causal=causal)


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("R", [2, 70])
def test_attend_scales(built_lib, cuda, dtype, R):
    for scale in (1e-3, 2.0):
        check(gen(8), DT[dtype], 64, 2, 2, 16, R, [50, 120], [R, R - 1], scale=scale)
        check(gen(8), DT[dtype], 64, 2, 2, 16, R, [50, 120] * 10, [R, R - 1] * 10, scale=scale)
    # groups whose scales lie far apart
    check(gen(9), DT[dtype], 64, 2, 2, 16, R, [50, 320], [R, R - 1], spread=20, scale=0.01)
    check(gen(9), DT[dtype], 64, 2, 2, 16, R, [50, 320] * 10, [R, R - 1] * 10, spread=20, scale=0.01)


def test_attend_one_long_sequence(built_lib, cuda):
    """Every head split over many warps and joined."""
    check(gen(10), DT["bf16"], 64, 2, 1, 16, 3, [20011], [3])
    check(gen(10), DT["fp16"], 128, 8, 1, 64, 1, [20011], [1])


def test_attend_many_sequences(built_lib, cuda):
    lens = [(i * 37) % 90 for i in range(70)]
    check(gen(11), DT["bf16"], 64, 2, 2, 16, 2, lens, [i % 3 for i in range(70)])


@pytest.mark.parametrize("dtype,dim,R", [("bf16", 64, 2), ("bf16", 64, 11), ("fp16", 128, 9)])
def test_attend_long_among_many_short(built_lib, cuda, dtype, dim, R):
    lens = [3] * 150 + [9001] + [5] * 140
    check(gen(16), DT[dtype], dim, 1, 1, 16, R, lens, [R] * 150 + [R] + [1] * 140)


def test_attend_most_sequences(built_lib, cuda):
    check(gen(17), DT["bf16"], 64, 1, 1, 16, 1, [(i * 5) % 40 for i in range(1024)], [i % 2 for i in range(1024)])


@pytest.mark.parametrize("R", [4, 80])
def test_a_hidden_nan_does_not_reach_a_row(built_lib, cuda, R):
    """NaN and infinities among the new rows become NaN codes: rows before them do not see them, later ones are NaN."""
    def spoil(q, kn, vn, v, vs, table):
        vn[0, 2, 0, 3], vn[1, 1, 1, 60], kn[2, 3, 0, 5] = math.nan, math.inf, -math.inf
    check(gen(12), DT["bf16"], 64, 4, 2, 16, R, [0, 14, 29, 61], [R, R, R, R - 1], spoil=spoil)
    check(gen(12), DT["bf16"], 64, 4, 2, 16, R, [0, 14, 29, 61] * 5, [R, R, R, R - 1] * 5, spoil=spoil)


@pytest.mark.parametrize("dtype", ["fp16", "bf16"])
@pytest.mark.parametrize("R", [1, 70])
def test_scales_that_are_no_powers_of_two(built_lib, cuda, R, dtype):
    """A cache quantised elsewhere: scales of any value, groups of zeros with the least scale, one group with a huge one."""
    def spoil(q, kn, vn, v, vs, table):
        ok = torch.isfinite(vs)
        vs[ok] *= 1.37
        v[int(table[1, 0])] = torch.zeros_like(v[int(table[1, 0])].float()).to(v.dtype)
        vs[int(table[1, 0])] = 2.0 ** -126
        vs[int(table[1, 1]), 0, 0] = 2.0 ** 30
    check(gen(13), DT[dtype], 64, 4, 2, 16, R, [64, 96], [R, R], causal=False, spoil=spoil)
    check(gen(13), DT[dtype], 64, 4, 2, 16, R, [64, 96] * 10, [R, R] * 10, causal=False, spoil=spoil)


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("R", [1, 40])
def test_rows_of_wide_range(built_lib, cuda, dtype, R):
    """Rows of q that are zero, very small, or hold very large elements beside ordinary ones."""
    def spoil(q, kn, vn, v, vs, table):
        big = 3e4 if dtype == "fp16" else 1e30
        q[0] *= 0
        q[1] *= 1e-4 if dtype == "fp16" else 1e-30
        q[2, :, 0, :] *= 0
        q[2, :, 0, 1], q[2, :, 0, 2] = big, -big / 3
    scale = 1e-30 if dtype == "bf16" else 1e-4
    check(gen(14), DT[dtype], 64, 2, 2, 16, R, [40, 50, 60], [R, R, R], spoil=spoil, scale=scale)
    check(gen(15), DT[dtype], 64, 8, 2, 16, R, [40, 50, 60] * 7, [R, R, R] * 7, spoil=spoil, scale=scale)      # 4 heads a K/V head


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("dim,page", [(64, 16), (128, 48)])
def test_append_matches_plain(built_lib, cuda, dtype, dim, page):
    from paper_2608_12703_gb300 import serving
    g = gen(dim + page)
    lens, rows, R, K = [0, 1, 5, 15, 16, 17, 100, 31], [37, 0, 3, 1, 37, 36, 20, 2], 37, 3
    k, v, ks, vs, table = pool(g, K, dim, page, [n + R for n in lens])
    fill(g, k, ks, table, lens)
    fill(g, v, vs, table, lens)
    kn, vn = (randn(g, len(lens), R, K, dim).to(DT[dtype]) for _ in range(2))
    # exact edges of the scales, groups of zeros, values far beyond the group's own scale
    kn[0, 0] = 448.0
    kn[0, 1:17] = 0
    kn[0, 16:33, 1] = 1.75 * 2.0 ** -9
    vn[2, 0, :, 0] = 1.0e4
    vn[5, :, 0] *= 1e-4
    vn[6, 3, 1, 7] = math.nan
    if dtype != "fp16":
        vn[7, 1, 0, 0], vn[4, 0, 2] = 1e-38, 3e38
    kr, vr, ksr, vsr = k.clone(), v.clone(), ks.clone(), vs.clone()
    c = serving.PagedCache8(k, v, ks, vs, table)
    c.append(kn, vn, i32(lens), rows=i32(rows))
    assert c.status() == 0
    ref.append(kr, ksr, table, lens, rows, kn)
    ref.append(vr, vsr, table, lens, rows, vn)
    assert same_bits(ks, ksr) and same_bits(vs, vsr)
    assert torch.equal(codes(k), codes(kr)) and torch.equal(codes(v), codes(vr))


def test_append_in_pieces_keeps_what_a_group_holds(built_lib, cuda):
    """One row at a time: a group's scale only grows, and its earlier values stay within half a step of what they were."""
    from paper_2608_12703_gb300 import serving
    g = gen(31)
    k, v, ks, vs, table = pool(g, 2, 64, 16, [40])
    kr, vr, ksr, vsr = k.clone(), v.clone(), ks.clone(), vs.clone()
    c = serving.PagedCache8(k, v, ks, vs, table)
    for n in range(40):
        x, y = randn(g, 1, 1, 2, 64) * 2.0 ** (n % 7), randn(g, 1, 1, 2, 64)
        c.append(x, y, i32([n]))
        ref.append(kr, ksr, table, [n], [1], x)
        ref.append(vr, vsr, table, [n], [1], y)
    assert c.status() == 0
    assert torch.equal(codes(k), codes(kr)) and torch.equal(codes(v), codes(vr)) and same_bits(ks, ksr) and same_bits(vs, vsr)


@pytest.mark.parametrize("R", [2, 40, 400])
def test_data_errors(built_lib, cuda, R):
    """Lengths and page ids out of range leave their sequence zero (or read page 0), set the status, and touch nothing else."""
    from paper_2608_12703_gb300 import serving
    g = gen(20)
    lens, rows = [20, 20, 20, 20, 20], [R, R + 1, R, R, R]
    k, v, ks, vs, table = pool(g, 2, 64, 16, [n + R for n in lens])
    fill(g, k, ks, table, lens)
    fill(g, v, vs, table, lens)
    q, kn, vn = make_rows(g, 5, R, 8, 2, 64, torch.bfloat16, True)      # of 400 rows 7 tiles a head: the kernel for prompts
    lens[2], lens[3] = -1, 16 * table.shape[1] - R + 1
    table[4, 1] = 10 ** 6
    before = codes(k).clone()
    c = serving.PagedCache8(k, v, ks, vs, table)
    out, lse = c.attend(q, i32(lens), k_new=kn, v_new=vn, rows=i32(rows))
    assert c.status() == A.ST_BAD_LENS | A.ST_CAPACITY | A.ST_BOUNDS
    assert c.status() == 0
    assert bool((out[1:4] == 0).all()) and bool((lse[1:4] == -math.inf).all())
    own = set(table[0].tolist()) | set(table[4, 2:].tolist())
    others = [p for p in range(k.shape[0]) if p not in own]
    assert torch.equal(codes(k)[others], before[others])


def test_side_stream_and_graph(built_lib, cuda):
    from paper_2608_12703_gb300 import serving
    g = gen(21)
    lens, R = [40, 100, 7], 3
    k, v, ks, vs, table = pool(g, 2, 64, 16, [n + R for n in lens])
    fill(g, k, ks, table, lens)
    fill(g, v, vs, table, lens)
    q, kn, vn = make_rows(g, 3, R, 4, 2, 64, torch.bfloat16, True)
    c = serving.PagedCache8(k, v, ks, vs, table)
    n = i32(lens)
    want = c.attend(q, n, k_new=kn, v_new=vn)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        other = c.attend(q, n, k_new=kn, v_new=vn)
    torch.cuda.current_stream().wait_stream(s)
    assert same_bits(want[0], other[0]) and same_bits(want[1], other[1])
    graph = torch.cuda.CUDAGraph()
    out, lse = torch.empty_like(want[0]), torch.empty_like(want[1])
    with torch.cuda.graph(graph):
        c.attend(q, n, k_new=kn, v_new=vn, out=out, lse=lse)
    q *= -1
    want = c.attend(q, n, k_new=kn, v_new=vn)
    for _ in range(3):
        out.zero_()
        graph.replay()
        assert same_bits(want[0], out) and same_bits(want[1], lse)
    assert c.status() == 0


@pytest.mark.parametrize("bad", [
    dict(q=lambda a: a["q"].float()), dict(q=lambda a: a["q"][:, :, :3]), dict(q=lambda a: a["q"].cpu()), dict(k_new=lambda a: None),
    dict(k_new=lambda a: a["k_new"].half()), dict(kv_len=lambda a: a["kv_len"].long()), dict(kv_len=lambda a: a["kv_len"][:2]),
    dict(causal=lambda a: False), dict(rows=lambda a: a["rows"].float()), dict(scale=lambda a: 0.0), dict(scale=lambda a: math.nan),
    dict(out=lambda a: torch.empty_like(a["q"]).float()), dict(lse=lambda a: torch.empty(3, device="cuda")),
    dict(q=lambda a: a["q"].transpose(2, 3).contiguous().transpose(2, 3))], ids=lambda d: next(iter(d)))
def test_refusals(built_lib, cuda, bad):
    from paper_2608_12703_gb300 import serving
    g = gen(22)
    k, v, ks, vs, table = pool(g, 2, 64, 16, [40, 40, 40])
    q, kn, vn = make_rows(g, 3, 2, 4, 2, 64, torch.bfloat16, False)
    c = serving.PagedCache8(k, v, ks, vs, table)
    a = dict(q=q, kv_len=i32([3, 4, 5]), k_new=kn, v_new=vn, rows=i32([1, 2, 0]), causal=True)
    (name, make), = bad.items()
    a[name] = make(a)
    with pytest.raises(A.AsrSpecError, match="INVAL"):
        c.attend(a.pop("q"), a.pop("kv_len"), **a)


def test_cache_refusals(built_lib, cuda):
    from paper_2608_12703_gb300 import serving
    k, v, ks, vs, table = pool(gen(23), 2, 64, 32, [40])
    serving.PagedCache8(k, v, ks, vs, table)
    for a in ((k.cpu(), v, ks, vs, table), (k.float(), v.float(), ks, vs, table), (k, v[1:], ks, vs, table),
              (k, v, ks[:, :, :1], vs, table), (k, v, ks.double(), vs, table), (k, v, ks, vs.transpose(1, 2), table),
              (k, v, ks, vs, table.long()), (k[:, :, :24], v[:, :, :24], ks, vs, table), (k[..., :32], v[..., :32], ks, vs, table)):
        with pytest.raises(A.AsrSpecError, match="INVAL"):
            serving.PagedCache8(*a)


def test_calls_of_all_sizes_share_a_workspace(built_lib, cuda):
    """Few rows, prompts and single tokens in turn on one cache and stream: each finds the workspace as the one before left it."""
    from paper_2608_12703_gb300 import serving
    g = gen(24)
    lens = [700, 3, 90, 0]
    k, v, ks, vs, table = pool(g, 2, 64, 16, [n + 300 for n in lens])
    fill(g, k, ks, table, [n + 300 for n in lens])
    fill(g, v, vs, table, [n + 300 for n in lens])
    c = serving.PagedCache8(k, v, ks, vs, table)
    want = {}
    for turn in range(3):
        for R in (1, 300, 7, 40, 129):
            q = torch.randn((4, R, 8, 64), generator=gen(R), device="cuda").half()
            n = i32([x + 300 - R for x in lens])
            got = c.attend(q, n)
            if turn == 0:
                want[R] = got
                compare(*got, *ref.attend(q, k, v, ks, vs, table, [x + 300 - R for x in lens], [R] * 4, True, 0.125))
            assert same_bits(got[0], want[R][0]) and same_bits(got[1], want[R][1])
    assert c.status() == 0


@pytest.mark.parametrize("R,heads", [(2, 2), (70, 2), (300, 20)])
def test_offsets_past_32_bits(built_lib, cuda, R, heads):
    """A pool of more than 4 GB, the sequences in its last pages."""
    from paper_2608_12703_gb300 import serving
    g, page, K = gen(25), 16, 1
    n_pages = (9 << 29) // (page * 64)      # 4.5 GiB of codes each
    k, v = (torch.empty((n_pages, K, page, 64), dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn) for _ in range(2))
    ks, vs = (torch.empty((n_pages, K, 1), device="cuda") for _ in range(2))
    lens = [37, 200]
    need = [-(-(n + R) // page) for n in lens]
    ids = [n_pages - 1 - i for i in range(sum(need))]
    table = torch.zeros((2, max(need)), dtype=torch.int32, device="cuda")
    table[0, :need[0]], table[1, :need[1]] = i32(ids[:need[0]]), i32(ids[need[0]:])
    fill(g, k, ks, table, lens)
    fill(g, v, vs, table, lens)
    low, small = min(ids), table - min(ids)      # the same pages alone
    kr, vr, ksr, vsr = (x[low:].clone() for x in (k, v, ks, vs))
    q, kn, vn = make_rows(g, 2, R, heads, K, 64, torch.bfloat16, True)      # (300, 20): the kernel for prompts
    ref.append(kr, ksr, small, lens, [R, R], kn)
    ref.append(vr, vsr, small, lens, [R, R], vn)
    c = serving.PagedCache8(k, v, ks, vs, table)
    out, lse = c.attend(q, i32(lens), k_new=kn, v_new=vn)
    assert c.status() == 0
    assert torch.equal(codes(k[low:]), codes(kr)) and torch.equal(codes(v[low:]), codes(vr))
    compare(out, lse, *ref.attend(q, kr, vr, ksr, vsr, small, lens, [R, R], True, 0.125))


@pytest.mark.parametrize("R", [1, 20, 70])
@pytest.mark.parametrize("copies", [1, 10])
def test_scales_that_are_no_scales(built_lib, cuda, R, copies):
    """Scales that are zero stand for zeros; infinite, NaN and negative ones spoil no other sequence and end all the same."""
    from paper_2608_12703_gb300 import serving
    g = gen(26)
    lens = [100, 90, 80, 70, 60, 50] * copies
    k, v, ks, vs, table = pool(g, 2, 64, 16, lens)
    fill(g, k, ks, table, lens)
    fill(g, v, vs, table, lens)
    for b in range(0, len(lens), 6):
        vs[int(table[b, 1])], ks[int(table[b + 1, 1])] = math.nan, math.inf
        vs[int(table[b + 2, 0])], vs[int(table[b + 3, 2])] = math.inf, -1.0
        ks[int(table[b + 4, 0])], vs[int(table[b + 4, 1])] = 0.0, 0.0
    q = make_rows(g, len(lens), R, 4, 2, 64, torch.bfloat16, True)[0]
    c = serving.PagedCache8(k, v, ks, vs, table)
    out, lse = c.attend(q, i32(lens), causal=False)
    assert c.status() == 0
    want = ref.attend(q, k, v, ks, vs, table, lens, [R] * len(lens), False, 0.125)
    good = [b for b in range(len(lens)) if b % 6 > 3]
    compare(out[good], lse[good], *(x[good] for x in want))
