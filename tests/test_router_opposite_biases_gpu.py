"""Groups whose best two experts have large biases of opposite sign: the sum of two is small, the roundings of its terms are not."""
import numpy as np
import pytest
import torch

import reference64 as R64
from paper_2608_07964_b200 import binding as B

pytestmark = pytest.mark.gpu


def near_pairs(rng, T, size, spread):
    """f32 logits [T, 4] and biases [4] of two groups of two experts whose biased scores add up to nearly the same."""
    a, b = spread * rng.uniform(1.0, 2.0, 2)
    bias = np.array([a, -a + 0.3, b, -b], np.float32)
    z = rng.normal(size=(T, 4)).astype(np.float32)
    score = lambda v: 1 / (1 + np.exp(-v.astype(np.float64)))  # noqa: E731
    gap = bias[:2].astype(np.float64).sum() - bias[2:].astype(np.float64).sum()
    # the last logit makes up for the rest, but for a few millionths; tokens for which none does keep theirs
    want = gap + score(z[:, 0]) + score(z[:, 1]) - score(z[:, 2]) + size * rng.uniform(-1, 1, T)
    ok = (want > 0.01) & (want < 0.99)
    z[ok, 3] = np.log(want[ok] / (1 - want[ok])).astype(np.float32)
    return z, bias


@pytest.mark.parametrize("spread", [0.5, 8.0, 64.0, 256.0, 1024.0, 1e5])
@pytest.mark.parametrize("layout", ["two_of_two", "eight_of_two", "two_of_32"])
def test_the_better_group_stays(layout, spread):
    """Sums of two that differ by less than 2e-5, from terms of `spread`; in groups of two, and in groups of 32 whose other experts are masked."""
    rng = np.random.default_rng(int(spread) + len(layout))
    T, E, n_group = {"two_of_two": (3000, 4, 2), "eight_of_two": (3000, 16, 8), "two_of_32": (3000, 64, 2)}[layout]
    z4, b4 = near_pairs(rng, T, 2e-5, spread)
    places = [3, 31, 32, 60] if layout == "two_of_32" else [0, 1, 2, 3]
    z, bias = rng.normal(size=(T, E)).astype(np.float32), np.full((1, E), -np.inf, np.float32)
    z[:, places], bias[0, places] = z4, b4
    if layout == "eight_of_two":
        bias[0, 4:] = -3.0 * spread - 10.0      # groups that are far behind
    step = B.MoEStep(1, E, 2, 0, 64, 64, 1, [0] * E, T)
    router = B.Router("sigmoid", torch.from_numpy(bias).cuda(), n_group, 1, 2)
    batch = B.Batch([0, T], [0])
    step.eb_route_scored(batch, router, torch.from_numpy(z).cuda())
    want, w = R64.route(z, bias, np.zeros(T, int), 2, True, n_group, 1, 2, 1, 1.0)
    got = step.topk_idx[:T].cpu().numpy()
    wrong = (got != want).any(1)
    assert not wrong.any(), f"{wrong.sum()} of {T}"
    assert len(np.unique(want[:, 0])) > 1           # both groups win somewhere
    assert np.allclose(step.topk_w[:T].cpu().numpy(), w, rtol=2.0 ** -17, atol=1e-37)


def test_a_pair_of_groups_told_apart_by_their_terms_roundings():
    """0.32203613 against 0.32203638 in exact arithmetic; term by term in 32 bits 0.32204056 against 0.32202910."""
    z = torch.tensor([[-1.00223827, -0.19635658, 0.36778218, 1.92614210]], device="cuda")
    bias = torch.tensor([[63.80789566, -64.20542908, 65.33184052, -66.47354889]], device="cuda")
    step = B.MoEStep(1, 4, 2, 0, 64, 64, 1, [0] * 4, 1)
    step.eb_route_scored(B.Batch([0, 1], [0]), B.Router("sigmoid", bias, 2, 1, 2), z)
    assert step.topk_idx[0].tolist() == [2, 3]
