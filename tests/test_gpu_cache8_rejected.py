"""What rows that are appended and not committed leave behind in a group of an 8-bit cache."""
import pytest
import torch

from test_gpu_cache8 import gen, i32, pool, randn

pytestmark = pytest.mark.gpu


def values(pages, scales):
    return pages.double() * scales.double().repeat_interleave(16, dim=2)[..., None]


@pytest.mark.parametrize("R", [1, 6])
def test_committed_slots_after_rejected_drafts(built_lib, cuda, R):
    """Rounds of drafts of any size of which few stay.  A slot is rounded anew only where a scale grows by a power of two, to steps
    of 2^-9 of it below 2^-6 of it, by half a step at most: over all growths less than 2^-10 (1 + 1/2 + ..) = 2^-9 of the scale at
    the end.  Scales never shrink, and are those of the largest value that the group was given."""
    from paper_2608_12703_gb300 import serving
    g, K = gen(70), 3
    k, v, ks, vs, table = pool(g, K, 64, 32, [400])
    c = serving.PagedCache8(k, v, ks, vs, table)
    order = table[0].long()
    n, sure = 0, torch.empty((0, K, 64), dtype=torch.float64, device="cuda")      # the slots as they were when they were committed
    while n < 380:
        size = torch.exp2(torch.randint(-6, 14, (1, R, K, 1), generator=g, device="cuda").float())
        x, y = randn(g, 1, R, K, 64) * size, randn(g, 1, R, K, 64)
        old = ks[order].permute(1, 0, 2).reshape(K, -1)[:, :-(-n // 16)].clone()
        c.append(x, y, i32([n]))
        now = values(k[order], ks[order]).permute(0, 2, 1, 3).reshape(-1, K, 64)
        s = ks[order].permute(1, 0, 2).reshape(K, -1)
        assert bool((s[:, :old.shape[1]] >= old).all())
        per_slot = s.repeat_interleave(16, dim=1).T[:n, :, None].double()
        off = (now[:n] - sure[:n]).abs()
        assert bool((off <= 2.0 ** -9 * per_slot).all())
        # values that are normal under the scale are as they were
        same = sure[:n].abs() >= 2.0 ** -6 * per_slot
        assert torch.equal(now[:n][same], sure[:n][same])
        m = int(torch.randint(0, R + 1, (1,), generator=g, device="cuda")) if R > 1 else int(torch.rand(1, generator=g, device="cuda") < 0.5)
        sure = torch.cat([sure, now[n:n + m]])
        n += m
    assert c.status() == 0
