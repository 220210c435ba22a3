"""Caches in 8 bits whose scales share memory: they can be read, and nothing is appended to them."""
import itertools
import math
import random

import pytest
import torch

import cache8_ref as ref
import test_cache8_args as args
from paper_2608_12703_gb300 import asrspec as A

ref_ = args.ref


def appends(L, **kw):
    """What a call with new rows gets whose workspace is too small: refused for that alone where the cache may be written."""
    return L.asr_spec_paged8_attend(ref_(args.cache(**kw)), ref_(args.rows(heads=12)), 1, 4096, None, 4096, 0, None)


SHARED = [dict(scale_page_stride=0), dict(scale_head_stride=0), dict(scale_page_stride=0, scale_head_stride=0), dict(v_scale=256),
          dict(v_pages=4096), dict(scale_head_stride=1), dict(scale_page_stride=3), dict(v_scale=256 + 4), dict(v_scale=256 + 4 * 20),
          dict(k_scale=512, v_scale=256 + 4 * 30)]
OWN = [dict(), dict(v_scale=256 + 40 * 4), dict(k_scale=512, v_scale=256), dict(n_pages=1, scale_page_stride=0, max_pages=1),
       dict(kv_heads=1, scale_head_stride=0), dict(scale_page_stride=8, scale_head_stride=4, v_scale=256 + 2 * 4),
       dict(scale_page_stride=8, scale_head_stride=2, v_scale=256 + 4 * 4), dict(scale_head_stride=20, scale_page_stride=2),
       dict(page_size=16, scale_head_stride=2, v_scale=260)]


@pytest.mark.parametrize("shared", SHARED, ids=str)
def test_rows_are_not_appended_under_shared_scales(built_lib, shared):
    L, c = built_lib, ref_(args.cache(**shared))
    assert appends(L, **shared) == args.INVAL
    assert L.asr_spec_paged8_append(c, ref_(args.rows()), 1, None) == args.INVAL
    # reading goes on to the check of the workspace
    r = ref_(args.rows(k_new=None, v_new=None))
    assert L.asr_spec_paged8_attend(c, r, 1, 4096, None, 4096, 0, None) == args.CAPACITY
    assert L.asr_spec_paged8_attend_ws(c, r, 1) > 0


@pytest.mark.parametrize("own", OWN, ids=str)
def test_scales_of_their_own(built_lib, own):
    assert appends(built_lib, **own) == args.CAPACITY


def test_the_rule_against_a_list_of_addresses(built_lib):
    rng, seen = random.Random(3), {args.INVAL: 0, args.CAPACITY: 0}
    for _ in range(3000):
        pages, heads, groups = rng.randint(1, 5), rng.randint(1, 4), rng.randint(1, 3)
        sp, sh, apart = rng.randint(0, 20), rng.randint(0, 14), rng.randint(-40, 40)
        at = [p * sp + h * sh + g for p, h, g in itertools.product(range(pages), range(heads), range(groups))]
        want = args.CAPACITY if len(set(at + [x + apart for x in at])) == 2 * len(at) else args.INVAL
        seen[want] += 1
        got = appends(built_lib, n_pages=pages, kv_heads=heads, page_size=16 * groups, max_pages=1, k_scale=4096, v_scale=4096 + 4 * apart,
                      scale_page_stride=sp, scale_head_stride=sh)
        assert got == want, (pages, heads, groups, sp, sh, apart)
    assert min(seen.values()) > 300


@pytest.mark.parametrize("stride", [dict(scale_page_stride=1 << 40), dict(scale_head_stride=1 << 62)], ids=str)
def test_strides_past_any_memory(built_lib, stride):
    r = ref_(args.rows(k_new=None, v_new=None))
    assert built_lib.asr_spec_paged8_attend_ws(ref_(args.cache(**stride)), r, 1) == args.INVAL


def expanded(kind, pages, heads, groups):
    if kind == "all":
        return torch.full((1, 1, 1), 0.25, device="cuda").expand(pages, heads, groups)
    if kind == "pages":
        return torch.exp2(-torch.arange(heads * groups, device="cuda").float()).reshape(1, heads, groups).expand(pages, heads, groups)
    return torch.exp2(-torch.arange(pages * groups, device="cuda").float() % 5).reshape(pages, 1, groups).expand(pages, heads, groups)


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["all", "pages", "heads", "k is v"])
@pytest.mark.parametrize("R", [2, 300])
def test_reading_under_shared_scales(built_lib, cuda, kind, R):
    from paper_2608_12703_gb300 import serving
    from test_gpu_cache8 import codes, compare, fill, gen, i32, make_rows, pool
    g, lens, K, page = gen(40), [70, 33, 0, 200], 20, 16 if kind == "all" else 32
    k, v, ks, vs, table = pool(g, K, 64, page, [n + R for n in lens])
    fill(g, k, ks.clone(), table, [n + R for n in lens])
    fill(g, v, vs.clone(), table, [n + R for n in lens])
    if kind == "k is v":
        ks = vs = torch.exp2(torch.randint(-8, 0, ks.shape, generator=g, device="cuda").float())
    else:
        ks, vs = expanded(kind, *ks.shape), expanded(kind, *ks.shape)
    q, kn, vn = make_rows(g, len(lens), R, K, K, 64, torch.bfloat16, True)
    c = serving.PagedCache8(k, v, ks, vs, table)
    out, lse = c.attend(q, i32(lens))      # the rows' K/V are in the pages
    compare(out, lse, *ref.attend(q, k, v, ks, vs, table, lens, [R] * 4, True, 1 / math.sqrt(64)))
    before, scales = codes(k).clone(), ks.clone()
    with pytest.raises(A.AsrSpecError, match="of their own"):
        c.attend(q, i32(lens), k_new=kn, v_new=vn)
    with pytest.raises(A.AsrSpecError, match="of their own"):
        c.append(kn, vn, i32(lens))
    pool_args = (c, i32([0] * 4), i32([0] * (k.shape[0] - 1) + [1]))
    if kind != "k is v":
        with pytest.raises(A.AsrSpecError, match="of their own"):
            serving.PagePool(*pool_args)
    else:      # the same scales for K and V move with their page
        last = codes(k[-1:]).clone(), ks[-1:].clone()
        serving.PagePool(*pool_args).compact()
        assert torch.equal(codes(k[:1]), last[0]) and torch.equal(ks[:1], last[1])
        before[:1], scales[:1] = last
    assert torch.equal(codes(k), before) and torch.equal(ks, scales) and c.status() == 0


@pytest.mark.gpu
def test_interleaved_scales_are_appended_under(built_lib, cuda):
    """K's and V's scales side by side in one array are each their own."""
    from paper_2608_12703_gb300 import serving
    from test_gpu_cache8 import codes, gen, i32, make_rows, pool, same_bits
    g, lens, R = gen(41), [0, 0], 20
    k, v, ks, vs, table = pool(g, 2, 64, 32, [R, R])
    both = torch.zeros((*ks.shape[:2], 2, ks.shape[2]), device="cuda")
    _, kn, vn = make_rows(g, 2, R, 2, 2, 64, torch.float16, True)
    kr, vr, ksr, vsr = k.clone(), v.clone(), torch.zeros_like(ks), torch.zeros_like(vs)
    c = serving.PagedCache8(k, v, both[:, :, 0], both[:, :, 1], table)
    c.append(kn, vn, i32(lens))
    ref.append(kr, ksr, table, lens, [R, R], kn)
    ref.append(vr, vsr, table, lens, [R, R], vn)
    assert c.status() == 0 and torch.equal(codes(k), codes(kr)) and torch.equal(codes(v), codes(vr))
    assert same_bits(both[:, :, 0], ksr) and same_bits(both[:, :, 1], vsr)
