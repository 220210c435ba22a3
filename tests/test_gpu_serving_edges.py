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
