"""Penalties, biases and masks on logits against a plain 64-bit implementation."""
import math

import numpy as np
import pytest
import torch

import cache8_ref as ref
from paper_2608_12703_gb300 import asrspec as A
from serving_ref import EPS_OUT

pytestmark = pytest.mark.gpu

DT = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}


def dev(x, dtype=None):
    return None if x is None else torch.tensor(np.asarray(x), dtype=dtype, device="cuda")


def inputs(seed, B, R, V, T, dtype, bias=None, mask=False):
    rng = np.random.default_rng(seed)
    x = torch.tensor(rng.normal(size=(B, R, V)) * 4, dtype=torch.float32).to(dtype)
    some = max(1, V // 20)
    a = dict(logits=x.float().numpy(), history=rng.integers(0, some, (B, T)), draft=rng.integers(0, some, (B, R - 1)),
             seen=rng.integers(0, T + 1, B), lens=np.array([R - 1 if b % 3 else rng.integers(-1, R) for b in range(B)]),
             rep=np.float32(1 + rng.random(B)), freq=np.float32(rng.normal(size=B)), pres=np.float32(rng.normal(size=B)), bias=None,
             mask=None)
    a["prompt"] = np.array([rng.integers(0, n + 1) for n in a["seen"]])
    if bias:
        a["bias"] = np.float32(rng.normal(size=V if bias == 1 else (B, V)))
        a["bias"][..., rng.integers(0, V, max(1, V // 9))] = -np.inf
    if mask:
        a["mask"] = rng.integers(-2 ** 31, 2 ** 31, (B, R, -(-V // 32)), dtype=np.int64).astype(np.int32)
    return a, x


def call(a, x, out=None, status=None, **kw):
    from paper_2608_12703_gb300 import serving
    i = torch.int32
    args = dict(history=dev(a["history"], i), history_len=dev(a["seen"], i), prompt_len=dev(a["prompt"], i), draft=dev(a["draft"], i),
                lens=dev(a["lens"], i), repetition=dev(a["rep"]), frequency=dev(a["freq"]), presence=dev(a["pres"]),
                bias=dev(a["bias"]), mask=dev(a["mask"]), out=out, status=status)
    args.update(kw)
    return serving.adjust_logits(x, **args)


def compare(got, a, dtype, before):
    want, bound = ref.adjust(a["logits"], a["history"], a["seen"], a["prompt"], a["draft"], a["lens"], a["rep"], a["freq"], a["pres"],
                             a["bias"], a["mask"])
    got = got.double().cpu().numpy()
    use = ~np.isnan(bound) | np.isinf(want)
    rows = np.arange(want.shape[1])[None, :] <= np.asarray(a["lens"])[:, None]
    assert (got[~rows] == before[~rows]).all()      # rows past lens are left as they are
    fin = np.isfinite(want) & rows[..., None]
    inf = np.isinf(want) & rows[..., None]
    assert (got[inf] == want[inf]).all()
    # the type's rounding of the result: half a step (a subnormal fp16 one 2^-25), of a value off by the bound
    err = np.abs(got[fin] - want[fin])
    tol = bound[fin] + EPS_OUT[dtype] * (np.abs(want[fin]) + bound[fin]) + (2.0 ** -25 if dtype == torch.float16 else 0)
    assert (err <= tol).all(), (err / tol).max()
    assert use[rows].all()


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("B,R,V,T", [(1, 1, 1, 1), (1, 9, 51866, 200), (3, 4, 999, 17), (2, 32, 5000, 3000), (5, 2, 1024, 448),
                                     (2, 7, 51865, 40), (4, 3, 4100, 1), (2, 5, 2050, 300)])
def test_matches_plain(built_lib, cuda, dtype, B, R, V, T):
    for bias, mask in ((None, False), (1, True), (2, False), (None, True)):
        a, x = inputs(B + R + V + T, B, R, V, T, DT[dtype], bias, mask)
        x = x.cuda()
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        before = x.double().cpu().numpy()
        out = torch.full_like(x, 5.0)
        assert call(a, x, out, status) is out
        compare(out, a, DT[dtype], np.full_like(before, 5.0))
        assert np.array_equal(x.double().cpu().numpy(), before)
        assert call(a, x, None, status) is x      # in place
        compare(x, a, DT[dtype], before)
        assert int(status) == 0


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_strides(built_lib, cuda, dtype):
    """Rows at every alignment, in a wider array; histories, masks and biases that are slices too."""
    for V, pad in ((700, 0), (700, 1), (701, 3), (704, 8), (702, 2)):
        a, x = inputs(V + pad, 3, 4, V, 30, DT[dtype], 2, True)
        wide = torch.zeros((3, 5, V + pad), dtype=DT[dtype], device="cuda")
        view = wide[:, 1:, pad:] if pad else wide[:, 1:]
        view.copy_(x)
        out = torch.full((3, 4, V + pad + 1), 9.0, dtype=DT[dtype], device="cuda")
        hist = torch.zeros((3, 50), dtype=torch.int32, device="cuda")
        hist[:, 5:35] = dev(a["history"], torch.int32)
        bias = torch.zeros((3, V + 5), device="cuda")
        bias[:, 2:V + 2] = dev(a["bias"])
        mask = torch.zeros((3, 4, a["mask"].shape[2] + 3), dtype=torch.int32, device="cuda")
        mask[:, :, 1:-2] = dev(a["mask"])
        call(a, view, out[:, :, :V], history=hist[:, 5:35], bias=bias[:, 2:V + 2], mask=mask[:, :, 1:-2])
        compare(out[:, :, :V], a, DT[dtype], np.full((3, 4, V), 9.0))
        assert bool((out[:, :, V:] == 9.0).all())


@pytest.mark.parametrize("V", [77, 3001])
def test_defaults_and_numbers(built_lib, cuda, V):
    """Each argument left out; one number for all."""
    from paper_2608_12703_gb300 import serving
    a, x = inputs(V, 3, 4, V, 20, torch.float32)
    x = x.cuda()
    assert torch.equal(serving.adjust_logits(x, out=torch.empty_like(x)), x)
    a.update(lens=np.full(3, 3), seen=np.full(3, 20), prompt=np.zeros(3, int), rep=np.full(3, np.float32(1.3)), freq=np.full(3, np.float32(0.5)),
             pres=np.full(3, np.float32(-0.25)))
    out = torch.empty_like(x)
    call(a, x, out, lens=None, history_len=None, prompt_len=None, repetition=1.3, frequency=0.5, presence=-0.25)
    compare(out, a, torch.float32, a["logits"])
    a["history"] = np.zeros((3, 0), int)
    a["seen"] = np.zeros(3, int)
    call(a, x, out, lens=None, history=None, history_len=None, prompt_len=None)
    compare(out, a, torch.float32, a["logits"])
    call(a, x, out)      # a history without room
    compare(out, a, torch.float32, a["logits"])
    a["draft"] = np.full((3, 3), -1)      # no drafts at all
    call(a, x, out, draft=None, lens=None)
    compare(out, a, torch.float32, a["logits"])


@pytest.mark.parametrize("dtype", ["fp32", "fp16"])
def test_numbers_that_are_not_finite(built_lib, cuda, dtype):
    """Infinite and NaN logits stay what they are but where the mask forbids them; a row may be masked whole."""
    a, x = inputs(3, 2, 3, 500, 40, DT[dtype], None, True)
    a["freq"] = np.abs(a["freq"])
    x[0, 0, :40], x[0, 1, :40], x[1, 1, :40] = math.inf, -math.inf, math.nan
    a["mask"][1, 2] = 0
    a["mask"][0, 0, 0] = 1
    a["lens"] = np.array([2, 2])
    got = call(a, x.cuda(), torch.empty_like(x.cuda())).double().cpu().numpy()
    bits = np.unpackbits(np.ascontiguousarray(a["mask"]).view(np.uint8), bitorder="little").reshape(2, 3, -1)[..., :500].astype(bool)
    assert np.isneginf(got[~bits]).all()
    assert np.isposinf(got[0, 0, :40][bits[0, 0, :40]]).all() and np.isneginf(got[0, 1, :40]).all()
    assert np.isnan(got[1, 1, :40][bits[1, 1, :40]]).all()
    assert np.isneginf(got[1, 2]).all() and bits[0, 0, 0] and not bits[0, 0, 1:32].any()


def test_data_errors(built_lib, cuda):
    a, x = inputs(4, 6, 4, 300, 20, torch.float32)
    a["lens"] = np.array([3, 4, -2, 3, 3, 3])
    a["seen"] = np.array([20, 20, 20, 21, 20, 20])
    a["prompt"] = np.array([0, 0, 0, 0, -1, 3])
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    out = torch.full_like(x.cuda(), 5.0)
    call(a, x.cuda(), out, status)
    assert int(status) == A.ST_BAD_LENS and bool((out[1:5] == 5.0).all())
    keep = {k: v if v is None else v[[0, 5]] for k, v in a.items()}
    compare(out[[0, 5]], keep, torch.float32, np.full((2, 4, 300), 5.0))
    # tokens outside the vocabulary are passed over, wherever they stand
    a["lens"], a["seen"], a["prompt"] = np.full(6, 3), np.full(6, 20), np.full(6, 2)
    a["history"][0, 1], a["history"][2, 7], a["draft"][3, 2], a["draft"][4, 0] = -1, 300, 10 ** 9, -5
    status.zero_()
    call(a, x.cuda(), out, status)
    assert int(status) == A.ST_BAD_TOKEN
    compare(out, a, torch.float32, np.full((6, 4, 300), 5.0))


def test_side_stream_and_graph(built_lib, cuda):
    from paper_2608_12703_gb300 import serving
    a, x = inputs(5, 3, 5, 4000, 100, torch.float32, 1, True)
    x = x.cuda()
    want, out = torch.zeros_like(x), torch.zeros_like(x)
    i = torch.int32
    kw = {k: dev(a[n], i) for k, n in (("history", "history"), ("history_len", "seen"), ("prompt_len", "prompt"), ("draft", "draft"),
                                       ("lens", "lens"), ("mask", "mask"))}
    kw.update(repetition=dev(a["rep"]), frequency=dev(a["freq"]), presence=dev(a["pres"]), bias=dev(a["bias"]))
    serving.adjust_logits(x, out=want, **kw)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        serving.adjust_logits(x, out=out, **kw)
    torch.cuda.current_stream().wait_stream(s)
    assert torch.equal(out, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        serving.adjust_logits(x, out=out, **kw)
    x.neg_()
    serving.adjust_logits(x, out=want, **kw)
    out.zero_()
    graph.replay()
    assert torch.equal(out, want)


@pytest.mark.parametrize("bad", [
    dict(history=lambda a: a["history"].long()), dict(history=lambda a: None), dict(history=lambda a: a["history"].T),
    dict(history_len=lambda a: a["history_len"].float()), dict(prompt_len=lambda a: a["prompt_len"][:1]),
    dict(draft=lambda a: a["draft"][:, :1]), dict(lens=lambda a: a["lens"].cpu()), dict(repetition=lambda a: 0.0),
    dict(repetition=lambda a: "1"), dict(repetition=lambda a: a["repetition"].double()), dict(frequency=lambda a: math.nan),
    dict(presence=lambda a: math.inf), dict(bias=lambda a: torch.zeros(9, device="cuda")),
    dict(bias=lambda a: torch.zeros((2, 100), device="cuda").half()), dict(mask=lambda a: torch.zeros((2, 3, 3), dtype=torch.int32, device="cuda")),
    dict(out=lambda a: torch.zeros((2, 3, 100), device="cuda").half()), dict(status=lambda a: torch.zeros(2, dtype=torch.int32, device="cuda")),
    dict(frequency=lambda a: 1e38)], ids=lambda d: next(iter(d)))
def test_refusals(built_lib, cuda, bad):
    a, x = inputs(6, 2, 3, 100, 10, torch.float32)
    i = torch.int32
    kw = {k: dev(a[n], i) for k, n in (("history", "history"), ("history_len", "seen"), ("prompt_len", "prompt"), ("draft", "draft"),
                                       ("lens", "lens"))}
    kw.update(repetition=dev(a["rep"]), frequency=dev(a["freq"]), presence=dev(a["pres"]))
    (name, make), = bad.items()
    kw[name] = make(kw)
    with pytest.raises(A.AsrSpecError, match="INVAL"):
        call(a, x.cuda(), **kw)


def test_refused_logits(built_lib, cuda):
    from paper_2608_12703_gb300 import serving
    x = torch.zeros((2, 3, 100), device="cuda")
    for y in (x.cpu(), x.double(), x[0], x.transpose(1, 2), x[:, :0], torch.zeros((1, 33, 8), device="cuda"),
              torch.zeros((2, 1, 100), device="cuda").expand(2, 3, 100), torch.zeros((1, 3, 100), device="cuda").expand(2, 3, 100)):
        with pytest.raises(A.AsrSpecError, match="INVAL"):
            serving.adjust_logits(y)
