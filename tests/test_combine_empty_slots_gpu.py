"""Aggregation of tokens with slots that have no row: whatever weight such a slot holds, it adds nothing."""
import pytest
import torch

from paper_2608_07964_b200 import binding as B

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("weight", [float("nan"), float("inf"), -1e30])
def test_the_weight_of_a_slot_without_a_row_counts_for_nothing(weight):
    T, E, K, S, H = 40, 6, 3, 1, 200
    step = B.MoEStep(2, E, K, S, H, 64, 2, [0, 0, 0, 1, 1, 1], T)
    batch = B.Batch([0, 25, T], [0, 1])
    gen = torch.Generator(device="cuda").manual_seed(3)
    z = torch.randn((T, E), generator=gen, device="cuda")
    z[4, 1:] = float("-inf")
    z[7] = float("-inf")
    step.x.copy_(torch.randn((T, H), generator=gen, device="cuda"))
    step.eb_route_scored(batch, B.Router("sigmoid"), z)
    step.eb_schedule(batch, 1, B.POLICY_ALL)
    step.eb_permute(batch)
    step.yp.copy_(torch.randn(step.yp.shape, generator=gen, device="cuda"))
    step.eb_combine(batch)
    want = step.out.clone()
    empty = step.pos[:T, :K] < 0
    assert int(empty.sum()) == 2 + 3
    step.topk_w[:T][empty] = weight
    step.out.fill_(7.0)
    step.eb_combine(batch)
    assert torch.equal(step.out, want) and bool(torch.isfinite(want.float()).all())
