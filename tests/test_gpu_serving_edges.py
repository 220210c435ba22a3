"""The operators over a paged cache where they can go wrong: values and arguments at the edges of what they accept."""
import math

import numpy as np
import pytest
import torch

import serving_ref as ref
from paper_2608_12703_gb300 import asrspec as A
from test_gpu_serving import DT, check_accept, fill, gen, i32, make_accept, pool, same_bits

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("B,V", [(300, 1), (300, 5), (1000, 33)])
def test_accept_shortest_rows(built_lib, cuda, dtype, B, V):
    """Blocks that have next to nothing to read exchange their results as soon as they start; the same over many calls."""
    from paper_2608_12703_gb300 import serving
    x = make_accept(70 + V, DT[dtype], B, 2, V, True, 1.0)
    want = check_accept(*x, 1.0)
    t, d, n, u, r, q = x
    for _ in range(50):
        got = serving.accept_sampled(t, d, n, u, r, draft_logits=q)
        assert all(torch.equal(a, b) for a, b in zip(want, got))


@pytest.mark.parametrize("dim,R,G,n", [(64, 1, 1, 40000), (64, 3, 1, 40000), (64, 5, 4, 20000), (128, 1, 4, 40000), (128, 3, 4, 20000)])
def test_attend_long_tail_of_small_weights(built_lib, cuda, dim, R, G, n):
    """One strong key with a value of 0, and n keys of 2^-24 to 2^-27 of its weight with values of 1: their sum is the output."""
    from paper_2608_12703_gb300 import serving
    g = gen(71)
    k, v, table = pool(g, torch.float16, 1, dim, 256, [n + R])
    k.zero_()
    v.fill_(1.0)
    # slot 7 is the strong one: its score is 0, the others' -8 t with t in steps of 2^-6, exact in every type
    t = torch.randint(133, 150, (k.shape[0], 256), generator=g, device="cuda") / 64.0      # -8 t / ln 2: 2^-24.0 .. 2^-26.9
    k[:, 0, :, 0] = -t.half()
    at = (int(table[0, 0]), 0, 7)
    k[at], v[at] = 0.0, 0.0
    q = torch.zeros((1, R, G, dim), dtype=torch.float16, device="cuda")
    q[..., 0] = 8.0
    out, lse = serving.PagedCache(k, v, table).attend(q, i32([n]), scale=1.0)
    x = -8.0 * t[table[0].long()].double().reshape(-1)
    x[7] = 0.0
    for i in range(R):
        w = torch.exp(x[:n + i + 1])
        want, l = float((w.sum() - w[7]) / w.sum()), float(torch.log(w.sum()))
        # rounding of a weight and of the output to fp16, of exp2 and its argument, of a sum at every 16 keys
        rel = 2 * 2.0 ** -11 + 2.0 ** -20 * (1 + 19) + n / 16 * 2.0 ** -23
        assert float((out[0, i].double() - want).abs().max()) <= rel * want
        assert float((lse[0, i].double() - l).abs().max()) <= 2.0 ** -20 * (1 + 19)


@pytest.mark.parametrize("dim,kv_heads,B", [(64, 32, 60), (128, 16, 90)])
def test_attend_tail_of_small_weights_walked_by_one_warp(built_lib, cuda, dim, kv_heads, B):
    """The same with so many heads that nobody splits one: every weight is taken relative to the strong key's."""
    from paper_2608_12703_gb300 import serving
    g = gen(80)
    n, page = 1999, 400
    k, v, table = pool(g, torch.float16, kv_heads, dim, page, [n + 1] * B)
    k.zero_()
    v.fill_(64.0)
    t = torch.randint(133, 150, (k.shape[0], page), generator=g, device="cuda") / 64.0
    k[:, :, :, 0] = -t.half()[:, None, :]
    first = table[:, 0].long()
    k[first, :, 7], v[first, :, 7] = 0.0, 0.0
    q = torch.zeros((B, 1, kv_heads, dim), dtype=torch.float16, device="cuda")
    q[..., 0] = 8.0
    out, _ = serving.PagedCache(k, v, table).attend(q, i32([n] * B), scale=1.0)
    x = -8.0 * t[table.long()].double().reshape(B, n + 1)
    x[:, 7] = 0.0
    w = torch.exp(x)
    want = (64.0 * (w.sum(1) - w[:, 7]) / w.sum(1))[:, None, None, None]
    rel = 2 * 2.0 ** -11 + 2.0 ** -20 * (1 + 19) + n / 16 * 2.0 ** -23
    assert bool(((out.double() - want).abs() <= rel * want).all())


def test_attend_fp16_large_scores(built_lib, cuda):
    """Scores whose rounding is several powers of two: the weights stay in fp16's range, the strongest keys share the output."""
    from paper_2608_12703_gb300 import serving
    g = gen(72)
    k, v, table = pool(g, torch.float16, 2, 64, 16, [70])
    k.zero_()
    v.copy_(torch.randn(v.shape, generator=g, device="cuda"))
    k[:, :, :, 0] = -1.0
    for s in (3, 33, 64):       # the same largest score, about 2^35.5
        k[int(table[0, s // 16]), :, s % 16] = 60000.0
    q = torch.full((1, 2, 2, 64), 60000.0, dtype=torch.float16, device="cuda")
    q[:, :, 1] = 59968.0
    out, lse = serving.PagedCache(k, v, table).attend(q, i32([68]))
    vv = ref.slots(v, table[0], 70)
    want = vv[[3, 33, 64]].mean(0)[None, None].expand(1, 2, 2, 64)
    bound = 3 * 2.0 ** -11 * vv[[3, 33, 64]].abs().sum(0) + 2.0 ** -20
    assert bool(torch.isfinite(out).all()) and bool(torch.isfinite(lse).all())
    assert bool(((out.double() - want).abs() <= bound).all())


def test_numbers_given_as_tensors(built_lib, cuda):
    """A scale, causal flag, budget or temperature in a tensor is its value at the call, whatever an earlier call's was."""
    from paper_2608_12703_gb300 import serving
    g = gen(73)
    k, v, table = pool(g, torch.bfloat16, 2, 64, 16, [60, 60])
    fill(g, k, table, [60, 60])
    fill(g, v, table, [60, 60])
    q = torch.randn((2, 2, 4, 64), generator=g, device="cuda").bfloat16()
    n = i32([50, 33])
    c = serving.PagedCache(k, v, table)
    score = torch.rand((2, 2, 64), generator=g, device="cuda")
    fresh = lambda: serving.PagedCache(k.clone(), v.clone(), table)
    for scale in (0.5, 2.0, 0.125):
        for causal in (True, False):
            want, wl = fresh().attend(q, n, scale=scale, causal=causal)
            got, gl = c.attend(q, n, scale=torch.tensor(scale), causal=torch.tensor(causal))
            assert same_bits(got, want) and same_bits(gl, wl)
            ws = fresh().weigh(q, wl, n, score, scale=scale, causal=causal, out=torch.zeros_like(score))
            gs = c.weigh(q, wl, n, score, scale=torch.tensor(scale), causal=torch.tensor(causal), out=torch.zeros_like(score))
            assert torch.equal(gs, ws)
    pos = torch.arange(64, dtype=torch.int32, device="cuda").repeat(2, 2, 1).contiguous()
    for budget in (2, 30, 8):
        for recent in (0, 1):
            want = fresh().evict(n, score.clone(), pos.clone(), n, budget=budget, recent=recent)
            got = fresh_one(c, k, v).evict(n, score.clone(), pos.clone(), n, budget=torch.tensor(budget), recent=torch.tensor(recent))
            assert torch.equal(got[0], want[0])
            assert torch.equal(got[1][:, :, :budget], want[1][:, :, :budget]) and torch.equal(got[2][:, :, :budget], want[2][:, :, :budget])
    t, d, m, u, r, ql = make_accept(74, torch.float32, 4, 2, 100, True, 1.0)
    for temperature in (0.3, 2.0):
        want = serving.accept_sampled(t, d, m, u, r, draft_logits=ql, temperature=temperature)
        got = serving.accept_sampled(t, d, m, u, r, draft_logits=ql, temperature=torch.tensor(temperature))
        assert all(torch.equal(x, y) for x, y in zip(want, got))


def fresh_one(c, k, v):
    """The same cache object: its pages as they were, what it remembers kept."""
    c.k_pages.copy_(k)
    c.v_pages.copy_(v)
    return c


@pytest.mark.parametrize("inplace", [False, True])
@pytest.mark.parametrize("side", ["source", "destination"])
def test_evict_bad_page(built_lib, cuda, inplace, side):
    """A slot whose page id, or whose destination's, is out of range is not moved: not its K and V, score or position."""
    from paper_2608_12703_gb300 import serving
    g = gen(75)
    n, budget, page = 96, 40, 16
    k, v, table = pool(g, torch.bfloat16, 2, 64, page, [n, n])
    fill(g, k, table, [n, n])
    fill(g, v, table, [n, n])
    score = torch.rand((2, 2, n), generator=g, device="cuda")
    pos = torch.stack([torch.randperm(n, generator=g, device="cuda") for _ in range(4)]).view(2, 2, n).to(torch.int32)
    bad = table.clone()
    broken = 3 if side == "source" else 1          # slots 48 .. 63, or 16 .. 31, of the second sequence
    bad[1, broken] = k.shape[0] if side == "source" else -1
    k0, v0, s0, p0 = k.clone(), v.clone(), score.clone(), pos.clone()
    c = serving.PagedCache(k, v, bad)
    outs = {} if inplace else dict(score_out=torch.full((2, 2, budget), -5.0, device="cuda"),
                                   pos_out=torch.full((2, 2, budget), -5, dtype=torch.int32, device="cuda"))
    lens, so, po = c.evict(i32([n, n]), score, pos, i32([n, n]), budget=budget, **outs)
    assert c.status() == A.ST_BOUNDS and lens.tolist() == [budget, budget]
    plan = ref.evict([n, n], s0.cpu(), p0.cpu(), [n, n], budget, 0, 0)
    stuck = 0
    for b in range(2):
        for h in range(2):
            order = list(plan[b][h])
            for to, of in enumerate(order):
                if b == 1 and to != of and (to if side == "destination" else of) // page == broken:
                    order[to] = to
                    stuck += 1
            idx = torch.tensor(order, device="cuda")
            assert torch.equal(so[b, h, :budget], s0[b, h][idx]) and torch.equal(po[b, h, :budget], p0[b, h][idx])
            for new, old in ((k, k0), (v, v0)):
                a, o = ref.slots(new, table[b], n)[:, h], ref.slots(old, table[b], n)[:, h]
                assert torch.equal(a[:budget], o[idx]) and torch.equal(a[budget:], o[budget:])
    assert stuck > 0


def test_host_threads_share_a_cache(built_lib, cuda):
    """Threads that call one cache on one stream with growing sizes: every result as a cache of its own gives it."""
    import threading
    from paper_2608_12703_gb300 import serving
    g = gen(81)
    k, v, table = pool(g, torch.bfloat16, 2, 64, 16, [3000, 2900])
    fill(g, k, table, [3000, 2900])
    fill(g, v, table, [3000, 2900])
    n = i32([2900, 2800])
    qs = [torch.randn((2, r, 2 * h, 64), generator=g, device="cuda").bfloat16() for r, h in ((1, 1), (4, 2), (9, 1), (9, 4))]
    want = [serving.PagedCache(k, v, table).attend(q, n) for q in qs]
    torch.cuda.synchronize()
    for _ in range(5):
        c = serving.PagedCache(k, v, table)
        got, start = [[] for _ in qs], threading.Barrier(len(qs))

        def work(i):
            start.wait()
            for _ in range(20):
                got[i].append(c.attend(qs[i], n))
        threads = [threading.Thread(target=work, args=(i,)) for i in range(len(qs))]
        [t.start() for t in threads]
        [t.join() for t in threads]
        assert all(len(x) == 20 for x in got) and c.status() == 0
        for x, (out, lse) in zip(got, want):
            assert all(same_bits(a, out) and same_bits(b, lse) for a, b in x)


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("B,V", [(6, 51866), (20, 51865), (70, 51865), (9, 1003), (5, 8), (3, 300001)])
def test_accept_residual_of_equal_rows(built_lib, cuda, dtype, B, V):
    """Where p = q nothing is left of p - q: after a rejection (a drafted token masked in both) the token is drawn from p,
    whatever the rows' alignment."""
    t, _, _, u, r, _ = make_accept(76 + B, DT[dtype], B, 2, V, False, 0.8)
    d = torch.full((B, 2), V // 2, dtype=torch.int32, device="cuda")
    t[:, :, V // 2] = -math.inf
    x = (t, d, i32([2] * B), u, r, t[:, :2].contiguous())
    acc, tok, step, _ = check_accept(*x, 0.8)
    assert bool((acc == 0).all()) and bool((step == 1).all()) and bool((tok != V // 2).all())


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("dim", [64, 128])
def test_weigh_row_without_weight(built_lib, cuda, dtype, dim):
    """A row whose lse is -inf weighs nothing, also where its scores are infinite or NaN."""
    from paper_2608_12703_gb300 import serving
    g = gen(77)
    lens, R = [40, 7], 3
    k, v, table = pool(g, DT[dtype], 2, dim, 16, [n + R for n in lens])
    fill(g, k, table, [n + R for n in lens])
    v.zero_()
    q = torch.randn((2, R, 4, dim), generator=g, device="cuda").to(DT[dtype])
    c = serving.PagedCache(k, v, table)
    _, lse = c.attend(q, i32(lens))
    q[0, 1, :2], q[1, 0, 1], q[1, 2, 3] = math.inf, math.nan, -math.inf
    lse[0, 1, :2] = lse[1, 0, 1] = lse[1, 2, 3] = -math.inf
    out = c.weigh(q, lse, i32(lens), None, out=torch.full((2, 2, 48), -5.0, device="cuda"))
    want, bound = ref.weigh(q, lse, k, table, lens, [R, R], torch.zeros_like(out), True, 1 / math.sqrt(dim))
    live = ~torch.isnan(want)
    assert int(live.sum()) == 2 * sum(n + R for n in lens)
    assert bool(((out.double() - want).abs()[live] <= bound[live]).all())


def test_status_word_across_streams(built_lib, cuda):
    """The status word is clear before any stream's first call, and after it was read: what a call sets later stays."""
    from paper_2608_12703_gb300 import serving
    k, v = (torch.zeros((4, 2, 16, 64), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    table, q = i32([0, 1]).view(1, 2), torch.zeros((1, 1, 2, 64), dtype=torch.bfloat16, device="cuda")
    bad = i32([99])
    torch.cuda.synchronize()
    made, used = torch.cuda.Stream(), torch.cuda.Stream()
    with torch.cuda.stream(made):
        torch.cuda._sleep(200_000_000)          # the stream on which the cache is made is busy for 0.1 s
        c = serving.PagedCache(k, v, table)
    with torch.cuda.stream(used):
        c.attend(q, bad)
    assert c.status() == A.ST_CAPACITY
    for _ in range(20):
        with torch.cuda.stream(used):
            c.attend(q, bad)
        with torch.cuda.stream(made):
            assert c.status() == A.ST_CAPACITY
            assert made.query()                 # cleared already, not some time later


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("temperature", [1e-30, 3.5e-39, 4e-39, 1e-38, 1e30])
def test_accept_extreme_temperatures(built_lib, cuda, dtype, temperature):
    """From the row's maximum alone to every unmasked token alike."""
    from paper_2608_12703_gb300 import serving
    t, d, n, u, r, q = make_accept(78, torch.float32, 9, 3, 700, True, 1.0)
    t, q = t.clamp_(-8, 8).to(DT[dtype]), q.clamp_(-8, 8).to(DT[dtype])
    for x, rows in ((t, 4), (q, 3)):
        x[:, :, 5::9] = -math.inf
        x.scatter_(2, torch.randint(0, 700 // 9, (9, rows, 1), generator=gen(79), device="cuda") * 9, 9.0)
    d = t[:, :3].float().argmax(2).to(torch.int32)
    got = serving.accept_sampled(t, d, n, u, r, draft_logits=q, temperature=temperature)
    acc, tok, step, prob, _ = ref.accept(t.double().cpu().numpy(), d.cpu().numpy(), n.cpu().numpy(), u.double().cpu().numpy(),
                                         r.cpu().numpy(), q.double().cpu().numpy(), temperature)
    if temperature < 1:
        a, k, s, p = (x.cpu().numpy() for x in got)
        assert np.array_equal(a, acc) and np.array_equal(k, tok) and np.array_equal(s, step) and np.array_equal(p, prob)
    else:
        assert bool((got[1][n >= 0] >= 0).all()) and np.allclose(got[3].cpu().numpy(), prob, rtol=1e-5)


def test_arguments_of_other_kinds_are_refused(built_lib, cuda):
    """Lists and arrays in place of tensors, texts in place of numbers, whole numbers past 32 bits: an error of the package's
    own, before and after a call of the same layouts."""
    from paper_2608_12703_gb300 import serving
    z = lambda *s, dt=torch.bfloat16: torch.zeros(s, dtype=dt, device="cuda")
    c = serving.PagedCache(z(4, 2, 16, 64), z(4, 2, 16, 64), z(2, 2, dt=torch.int32))
    n, q = i32([8, 8]), z(2, 3, 4, 64)
    lse, s, p = z(2, 3, 4, dt=torch.float32), z(2, 2, 32, dt=torch.float32), z(2, 2, 32, dt=torch.int32)
    x = (z(2, 3, 9, dt=torch.float32), z(2, 2, dt=torch.int32), n, z(2, 2, dt=torch.float32), z(2, 9, dt=torch.float32) + 1)

    def refused(f):
        with pytest.raises(A.AsrSpecError, match="ASR_E_INVAL"):
            f()
    for _ in range(2):
        refused(lambda: c.attend(q, [8, 8]))
        refused(lambda: c.attend(q, n, rows=np.array([1, 1], dtype=np.int32)))
        refused(lambda: c.attend(None, n))
        refused(lambda: c.attend(q, n, scale="0.5"))
        refused(lambda: c.attend(q, n, scale=[0.5]))
        refused(lambda: c.attend(q, n, scale=torch.ones(2)))
        refused(lambda: c.weigh(q, lse, [8, 8], s))
        refused(lambda: c.weigh(q, lse.tolist(), n, s))
        refused(lambda: c.evict([8, 8], s, p, n, budget=4))
        refused(lambda: c.evict(n, s, p, n, budget=4.5))
        refused(lambda: c.evict(n, s, p, n, budget="4"))
        refused(lambda: c.evict(n, s, p, n, budget=(1 << 32) + 4))
        refused(lambda: c.evict(n, s, p, n, budget=4, recent=1 << 32))
        refused(lambda: c.evict(n, s, p, n, budget=4, first=1 << 31))
        refused(lambda: serving.accept_sampled(*x[:2], [2, 2], *x[3:]))
        refused(lambda: serving.accept_sampled(*x, temperature="1"))
        refused(lambda: serving.accept_sampled(*x, status=[0]))
        c.attend(q, n)
        c.weigh(q, lse, n, s)
        c.evict(n, s, p, n, budget=4, recent=(1 << 31) - 1, first=(1 << 31) - 1)
        serving.accept_sampled(*x)
    assert c.status() == 0


def one_head_attend(q, k, v, n, i, scale):
    """Row i of one head in 64 bits over the slots it sees: output, lse and their bounds (as serving_ref.attend's, of fp32
    sums of 16-bit products)."""
    kk, vv, qq = k[:n + i + 1].double(), v[:n + i + 1].double(), q.double()
    x = scale * (kk @ qq)
    l = torch.logsumexp(x, 0)
    p = torch.exp(x - l)
    ds = ref.score_bound(qq, kk, scale).max()
    rel = 2 * ds + 2.0 ** -20 * (1 + x.abs().max()) + (n + i + 1) * 2.0 ** -23
    return p @ vv, l, rel, p @ vv.abs(), ds + 2.0 ** -20 * (1 + l.abs() + x.abs().max())


@pytest.mark.parametrize("dtype,dim", [("bf16", 64), ("fp16", 128), ("fp32", 64)])
@pytest.mark.parametrize("lens,R,rows", [([0, 5, 100], 33, [33, 32, 7]), ([0, 3], 224, [224, 100]), ([1000], 1500, [1500]),
                                         ([64], 4096, [4096])])
def test_attend_prompt(built_lib, cuda, dtype, dim, lens, R, rows):
    """Prompts: many rows at once, into empty pages or behind others, two query heads on each K/V head."""
    from paper_2608_12703_gb300 import serving
    g = gen(82 + R)
    dt, K, G, page = DT[dtype], 2, 2, 80
    k, v, table = pool(g, dt, K, dim, page, [n + R for n in lens])
    fill(g, k, table, lens)
    fill(g, v, table, lens)
    qkv = torch.randn((len(lens), R, K * G + 2 * K, dim), generator=g, device="cuda").to(dt)
    q, kn, vn = qkv[:, :, :K * G], qkv[:, :, K * G:K * G + K], qkv[:, :, K * G + K:]
    c = serving.PagedCache(k, v, table)
    out, lse = c.attend(q, i32(lens), k_new=kn, v_new=vn, rows=i32(rows))
    assert c.status() == 0
    eps = ref.EPS_OUT[dt]
    for b, (n, r) in enumerate(zip(lens, rows)):
        ks, vs = (torch.cat([x[int(p)].transpose(0, 1) for p in table[b]])[:n + r] for x in (k, v))
        assert same_bits(ks[n:], kn[b, :r]) and same_bits(vs[n:], vn[b, :r])
        assert bool((out[b, r:] == 0).all()) and bool((lse[b, r:] == -math.inf).all())
        for h in range(K * G):
            for i in (i for i in sorted({0, 1, 15, 16, 31, 32, r // 2, r - 2, r - 1}) if i < r):
                want, l, rel, mass, lb = one_head_attend(q[b, i, h], ks[:, h // G], vs[:, h // G], n, i, dim ** -0.5)
                bound = (rel + (0.0 if dt == torch.float32 else eps)) * mass + 1.01 * eps * want.abs() + 2.0 ** -24
                assert bool(((out[b, i, h].double() - want).abs() <= bound).all())
                assert float((lse[b, i, h].double() - l).abs()) <= float(lb)


def test_weigh_data_errors(built_lib, cuda):
    """Bad lengths and rows and more slots than the scores have leave the sequence out; a bad page id is reported; the others
    are weighed."""
    from paper_2608_12703_gb300 import serving
    g = gen(83)
    k, v, table = pool(g, torch.bfloat16, 2, 64, 16, [48] * 3)
    fill(g, k, table, [48] * 3)
    v.zero_()
    q = torch.randn((3, 2, 2, 64), generator=g, device="cuda").bfloat16()
    lse = torch.full((3, 2, 2), 3.0, device="cuda")
    score = torch.rand((3, 2, 40), generator=g, device="cuda")
    c = serving.PagedCache(k, v, table)
    good = c.weigh(q, lse, i32([30] * 3), score, out=torch.full_like(score, -5.0))
    assert c.status() == 0
    for lens, rows, bit in (([30, 49, 30], [2, 2, 2], A.ST_CAPACITY), ([30, -1, 30], [2, 2, 2], A.ST_CAPACITY),
                            ([30, 47, 30], [2, 2, 2], A.ST_CAPACITY), ([30, 39, 30], [2, 2, 2], A.ST_CAPACITY),
                            ([30, 30, 30], [2, 3, 2], A.ST_BAD_LENS), ([30, 30, 30], [2, -1, 2], A.ST_BAD_LENS),
                            (None, [2, 2, 2], A.ST_BOUNDS)):
        t = table.clone()
        if lens is None:
            lens, t[1, 0] = [30] * 3, -3
        c = serving.PagedCache(k, v, t)
        pos = torch.full((3, 2, 40), -7, dtype=torch.int32, device="cuda")
        out = c.weigh(q, lse, i32(lens), score, rows=i32(rows), out=torch.full_like(score, -5.0), pos=pos, first_pos=i32([9] * 3))
        assert c.status() == bit and c.status() == 0
        assert torch.equal(out[0], good[0]) and torch.equal(out[2], good[2])
        if bit != A.ST_BOUNDS:
            assert bool((out[1] == -5.0).all()) and bool((pos[1] == -7).all())
        else:   # the other pages' slots as ever
            assert torch.equal(out[1, :, 16:32], good[1, :, 16:32])
        assert bool((out[:, :, 32:] == -5.0).all())


def test_operators_on_a_side_stream_and_in_a_graph(built_lib, cuda):
    """weigh, evict and accept_sampled on another stream, and replayed from a graph: the same results."""
    from paper_2608_12703_gb300 import serving
    g = gen(84)
    k, v, table = pool(g, torch.bfloat16, 4, 64, 16, [320, 100])
    fill(g, k, table, [320, 100])
    fill(g, v, table, [320, 100])
    q = torch.randn((2, 3, 8, 64), generator=g, device="cuda").bfloat16()
    lse = torch.full((2, 3, 8), 4.0, device="cuda")
    score = torch.rand((2, 4, 320), generator=g, device="cuda")
    pos = torch.arange(320, dtype=torch.int32, device="cuda").repeat(2, 4, 1).contiguous()
    n, new = i32([300, 90]), i32([303, 93])
    k0, v0 = k.clone(), v.clone()
    t, d, m, u, r, dl = make_accept(85, torch.float32, 5, 4, 20000, True, 1.0)
    c = serving.PagedCache(k, v, table)
    outs = dict(score_out=torch.zeros((2, 4, 64), device="cuda"), pos_out=torch.zeros((2, 4, 64), dtype=torch.int32, device="cuda"))
    out = torch.zeros_like(score)

    def calls():
        k.copy_(k0)
        v.copy_(v0)
        c.weigh(q, lse, n, score, out=out)
        lens, so, po = c.evict(new, out, pos, new, budget=64, recent=8, first=2, **outs)
        return [lens, *serving.accept_sampled(t, d, m, u, r, draft_logits=dl)]

    def results(x):
        torch.cuda.synchronize()
        return [y.clone() for y in x + [out[0, :, :303], out[1, :, :93], outs["score_out"], outs["pos_out"], k, v]]

    def clear(x):
        for y in x + [out, *outs.values(), k, v]:
            y.zero_()
    bits = lambda x: x.contiguous().view(torch.uint8)
    want = results(calls())
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        got = calls()
    assert all(torch.equal(bits(a), bits(b)) for a, b in zip(want, results(got)))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = calls()
    for _ in range(2):
        clear(got)
        graph.replay()
        assert all(torch.equal(bits(a), bits(b)) for a, b in zip(want, results(got)))
    assert c.status() == 0


def test_workspaces_grow(built_lib, cuda):
    """Calls of one cache that need more workspace than the ones before, and less again."""
    from paper_2608_12703_gb300 import serving
    g = gen(86)
    k, v, table = pool(g, torch.float16, 2, 128, 32, [5000, 4000])
    fill(g, k, table, [5000, 4000])
    fill(g, v, table, [5000, 4000])
    n = i32([4900, 3900])
    score = torch.rand((2, 2, 5000), generator=g, device="cuda")
    pos = torch.arange(5000, dtype=torch.int32, device="cuda").repeat(2, 2, 1).contiguous()
    c = serving.PagedCache(k, v, table)
    for R, G, budget in ((1, 1, 4890), (9, 4, 2500), (1, 1, 16), (17, 2, 3000)):
        q = torch.randn((2, R, 2 * G, 128), generator=g, device="cuda").half()
        got, want = c.attend(q, n), serving.PagedCache(k, v, table).attend(q, n)
        assert all(torch.equal(a, b) for a, b in zip(got, want))
        kk, vv, kw = k.clone(), v.clone(), dict(budget=budget, recent=5, first=1)
        got = c.evict(n, score.clone(), pos.clone(), n, **kw)
        want = serving.PagedCache(kk, vv, table).evict(n, score.clone(), pos.clone(), n, **kw)
        assert torch.equal(got[0], want[0]) and same_bits(k, kk) and same_bits(v, vv)
        assert torch.equal(got[1][:, :, :budget], want[1][:, :, :budget]) and torch.equal(got[2][:, :, :budget], want[2][:, :, :budget])


def test_binding_by_the_library_names(built_lib, cuda):
    """The functions of the binding with the library's names give what PagedCache and accept_sampled give."""
    import ctypes
    from paper_2608_12703_gb300 import serving
    g = gen(87)
    k, v, table = pool(g, torch.bfloat16, 2, 64, 16, [64, 64])
    fill(g, k, table, [64, 64])
    fill(g, v, table, [64, 64])
    q = torch.randn((2, 1, 4, 64), generator=g, device="cuda").bfloat16()
    n = i32([60, 33])
    c = serving.PagedCache(k, v, table)
    cache = A.AsrPagedCache(k.data_ptr(), v.data_ptr(), *k.stride()[:3], table.data_ptr(), table.stride(0), k.shape[0], 16,
                            table.shape[1], 2, 64, 2, 1, None)
    rows = A.AsrPagedRows(q.data_ptr(), *q.stride()[:3], None, None, 0, 0, 0, n.data_ptr(), None, 1, 4, 1, 0.125)
    ws = torch.zeros(built_lib.asr_spec_paged_attend_ws(ctypes.byref(cache), ctypes.byref(rows)), dtype=torch.uint8, device="cuda")
    want, wl = c.attend(q, n)
    out, lse = torch.zeros_like(want), torch.zeros_like(wl)
    stream = torch.cuda.current_stream().cuda_stream
    A.asr_spec_paged_attend(ctypes.byref(cache), rows, out, lse, ws, ws.numel(), stream)
    assert same_bits(out, want) and same_bits(lse, wl)
    score, pos = torch.rand((2, 2, 64), generator=g, device="cuda"), torch.arange(64, dtype=torch.int32, device="cuda").repeat(2, 2, 1).contiguous()
    ws_, got = c.weigh(q, lse, n, score, out=torch.zeros_like(score)), torch.zeros_like(score)
    s = A.AsrPagedScores(score.data_ptr(), None, 128, 64, 64, got.data_ptr(), None, 0, 0, 0, None)
    A.asr_spec_paged_weigh(ctypes.byref(cache), rows, s, lse, 4, 4, stream)
    assert torch.equal(got, ws_)
    kk, vv = k.clone(), v.clone()
    so, po, lo = torch.zeros((2, 2, 20), device="cuda"), torch.zeros((2, 2, 20), dtype=torch.int32, device="cuda"), torch.zeros_like(n)
    s = A.AsrPagedScores(score.data_ptr(), pos.data_ptr(), 128, 64, 64, so.data_ptr(), po.data_ptr(), 40, 20, 20, None)
    ws = torch.zeros(built_lib.asr_spec_paged_evict_ws(ctypes.byref(cache), ctypes.byref(s), 20), dtype=torch.uint8, device="cuda")
    A.asr_spec_paged_evict(ctypes.byref(cache), s, n, n, 20, 2, 1, lo, ws, ws.numel(), stream)
    want = serving.PagedCache(kk, vv, table).evict(n, score, pos, n, budget=20, recent=2, first=1, score_out=torch.zeros_like(so),
                                                   pos_out=torch.zeros_like(po))
    assert all(torch.equal(a, b) for a, b in zip((lo, so, po), want)) and same_bits(k, kk) and same_bits(v, vv)
    t, d, m, u, r, dl = make_accept(88, torch.float32, 3, 2, 500, True, 0.7)
    x = A.AsrSampledLogits(t.data_ptr(), *t.stride()[:2], dl.data_ptr(), *dl.stride()[:2], 3, 2, 500, 0)
    i = [torch.zeros(3, dtype=torch.int32, device="cuda") for _ in range(3)]
    prob = torch.zeros((3, 2), device="cuda")
    A.asr_spec_accept_sampled(x, d, m, u, r, r.stride(0), 0.7, *i, prob, None, stream)
    want = serving.accept_sampled(t, d, m, u, r, draft_logits=dl, temperature=0.7)
    assert all(torch.equal(a, b) for a, b in zip((*i, prob), want))


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("dim", [64, 128])
def test_attend_large_scores(built_lib, cuda, dtype, dim):
    """Scores of 2^35 and more, a little apart from their own rounding: the strongest keys share the output."""
    from paper_2608_12703_gb300 import serving
    g = gen(89)
    k, v, table = pool(g, DT[dtype], 2, dim, 16, [70])
    k.zero_()
    v.copy_(torch.randn(v.shape, generator=g, device="cuda"))
    k[:, :, :, 0] = -1.0
    for s in (3, 33, 64):       # the same largest score
        k[int(table[0, s // 16]), :, s % 16] = 59904.0
    q = torch.full((1, 2, 4, dim), 59904.0, dtype=DT[dtype], device="cuda")
    q[:, :, 1], q[:, :, 2] = 58880.0, 32768.0
    out, lse = serving.PagedCache(k, v, table).attend(q, i32([68]))
    vv = ref.slots(v, table[0], 70)[[3, 33, 64]]
    want = vv.mean(0).repeat_interleave(2, 0)[None, None].expand(1, 2, 4, dim)
    x = (59904.0 * dim * q[..., 0].double()) / math.sqrt(dim)
    eps = ref.EPS_OUT[DT[dtype]]
    bound = (eps + 2.0 ** -20) * vv.abs().sum(0).repeat_interleave(2, 0) + 1.01 * eps * want.abs() + 2.0 ** -24
    assert bool(((out.double() - want).abs() <= bound).all())
    assert bool(((lse.double() - x).abs() <= ((dim + 8) * 2.0 ** -22 + 2.0 ** -20) * x).all())
