"""Scores that are 1 or 0 alike in 64 bits: by the logits without a bias, ties (lowest index first) with one, of zeros too."""
import pytest
import torch

from paper_2608_07964_b200 import binding as B

pytestmark = pytest.mark.gpu


def choice(z, router, K=4):
    T, E = z.shape
    step = B.MoEStep(1, E, K, 0, 64, 64, 1, [0] * E, T)
    step.eb_route_scored(B.Batch([0, T], [0]), router, z)
    return step.topk_idx.long()


def logits(kind):
    """Twelve experts, a token with logits rising along them, one falling, one rising again."""
    up = torch.arange(12, device="cuda", dtype=torch.float32)
    z = torch.stack([up, up.flip(0), up.clone()])
    if kind == "softmax":
        z = -1000.0 - z            # far below the last expert, which takes all of the sum
        z[:, 11] = 0.0
    else:
        z += 40.0
    return z


def test_sigmoids_of_one():
    z = logits("sigmoid")
    zero = torch.zeros((1, 12), device="cuda")
    assert choice(z, B.Router("sigmoid")).tolist() == [[11, 10, 9, 8], [0, 1, 2, 3], [11, 10, 9, 8]]
    assert choice(z, B.Router("sigmoid", zero)).tolist() == [[0, 1, 2, 3]] * 3
    assert choice(z, B.Router("sigmoid", n_group=3, topk_group=1)).tolist() == [[11, 10, 9, 8], [0, 1, 2, 3], [11, 10, 9, 8]]
    assert choice(z, B.Router("sigmoid", zero, 3, 1)).tolist() == [[0, 1, 2, 3]] * 3
    assert choice(z, B.Router("sigmoid", n_group=3, topk_group=1, group_top=2)).tolist() == [[0, 1, 2, 3]] * 3      # a sum of two


def test_softmax_scores_of_zero():
    z = logits("softmax")
    zero = torch.zeros((1, 12), device="cuda")
    assert choice(z, B.Router("softmax")).tolist() == [[11, 0, 1, 2], [11, 10, 9, 8], [11, 0, 1, 2]]
    assert choice(z, B.Router("softmax", zero)).tolist() == [[11, 0, 1, 2]] * 3


@pytest.mark.parametrize("score", ["sigmoid", "softmax"])
def test_a_bias_of_zeros_changes_nothing_elsewhere(score):
    z = 3.0 * torch.randn((500, 48), generator=torch.Generator(device="cuda").manual_seed(1), device="cuda")
    zero = torch.zeros((1, 48), device="cuda")
    for groups in ((1, 1), (6, 2)):
        assert torch.equal(choice(z, B.Router(score, None, *groups)), choice(z, B.Router(score, zero, *groups)))
