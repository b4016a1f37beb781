"""Gating by scores, groups and a balance bias against the definition in 64 bits (and more): the choice exactly, the weights to 32 bits."""
import numpy as np
import pytest
import torch

import reference64 as R64
from paper_2608_07964_b200 import binding as B

pytestmark = pytest.mark.gpu


def make(E, K, tokens, L=3, D=4, renorm=1):
    off = [0] + np.cumsum(tokens).tolist()
    layers = [j % L for j in range(len(tokens))]
    step = B.MoEStep(L, E, K, 0, 64, 64, D, [e % D for e in range(E)], max(off[-1], 1), renorm_topk=renorm)
    layer_of = np.repeat(layers, tokens)
    return step, B.Batch(off, layers), layer_of


def check(step, batch, layer_of, z, router, bias, renorm, route=None):
    """z: the logits on the device, as they are handed over."""
    T, N, E, K = batch.n_tok, batch.n_mb, step.E, step.K
    idx, w = R64.route(z.double().cpu().numpy(), None if bias is None else bias.double().cpu().numpy(), layer_of, K, router.score == "sigmoid",
                       router.n_group, router.topk_group, router.group_top, renorm, router.scale)
    step.topk_idx.fill_(77), step.topk_w.fill_(-1.0), step.mb_load.fill_(9), step.mb_cnt.fill_(9)
    (route or (lambda: step.eb_route_scored(batch, router, z)))()
    got = step.topk_idx[:T].cpu().numpy()
    assert np.array_equal(got, idx), np.argwhere(got != idx)[:5]
    # exponentials, one quotient or two and a sum of at most 256 of them, in 32 bits
    assert np.allclose(step.topk_w[:T].cpu().numpy(), w, rtol=2.0 ** -17, atol=1e-37)
    cnt = np.zeros((N, E), int)
    for j in range(N):
        sel = idx[batch.tok_off[j]:batch.tok_off[j + 1]].reshape(-1)
        np.add.at(cnt[j], sel[sel >= 0], 1)
    load = np.zeros((N, step.D), int)
    np.add.at(load.T, [e % step.D for e in range(E)], cnt.T)
    assert np.array_equal(step.mb_cnt[:N].cpu().numpy(), cnt) and np.array_equal(step.mb_load[:N].cpu().numpy(), load)


def normal(shape, seed, sigma=1.0):
    return sigma * torch.randn(shape, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda")


GROUPS = [(64, 6, 1, 1), (64, 6, 8, 4), (256, 8, 8, 4), (60, 4, 5, 2), (33, 8, 3, 3), (7, 7, 7, 7), (1, 1, 1, 1), (32, 1, 32, 1), (96, 3, 32, 20), (250, 8, 10, 1)]


@pytest.mark.parametrize("renorm", [1, 0])
@pytest.mark.parametrize("with_bias", [True, False])
@pytest.mark.parametrize("score", ["sigmoid", "softmax"])
@pytest.mark.parametrize("E,K,n_group,topk_group", GROUPS)
def test_choice_and_weights(E, K, n_group, topk_group, score, with_bias, renorm):
    step, batch, layer_of = make(E, K, [37, 0, 1, 64, 5], renorm=renorm)
    z = normal((batch.n_tok, E), E + K, 2.0)
    bias = normal((3, E), 5, 0.3) if with_bias else None
    for group_top in (1, 2):
        router = B.Router(score, bias, n_group, topk_group, group_top, scale=2.5)
        check(step, batch, layer_of, z, router, bias, renorm)


@pytest.mark.parametrize("score", ["sigmoid", "softmax"])
@pytest.mark.parametrize("with_bias", [True, False])
def test_masked_experts_leave_slots_empty(score, with_bias):
    E, K = 24, 5
    step, batch, layer_of = make(E, K, [40, 33])
    z = normal((batch.n_tok, E), 8)
    drop = torch.rand(z.shape, generator=torch.Generator(device="cuda").manual_seed(1), device="cuda") < 0.75
    z[drop] = float("-inf")
    z[3], z[4] = float("-inf"), float("nan")         # nothing to choose from
    z[5, :20] = float("nan")
    z[6, 2], z[6, 9] = float("inf"), float("inf")    # counts as the largest float: a tie
    z[7], z[8] = -3.4e38, 3.4e38                     # the lowest and about the highest finite values: masks of that kind choose by index
    z[9], z[10] = -200.0, -1e4                       # scores that vanish, in 32 and in 64 bits
    bias = normal((3, E), 5, 0.1) if with_bias else None
    if with_bias:
        bias[1, 3], bias[1, 4], bias[0, 0] = float("-inf"), float("nan"), 100.0
    for n_group, topk_group, top in ((1, 1, 1), (4, 2, 2), (4, 1, 1), (24, 6, 2)):
        check(step, batch, layer_of, z, B.Router(score, bias, n_group, topk_group, top), bias, 1)


def test_empty_slots_have_no_rows_and_add_nothing():
    step, batch, _ = make(8, 3, [12, 9])
    step.bind_weights(*[normal((3, 8, 64, 64), i, 0.1).to(torch.bfloat16) for i in range(3)])
    z = normal((21, 8), 2)
    z[5], z[6, 1:], z[20] = float("-inf"), float("-inf"), float("nan")
    step.x.copy_(normal((21, 64), 3))
    step.logits.copy_(z)
    step.set_router(B.Router("sigmoid"))
    step.out.fill_(7.0)
    step.eb_step(batch, 1, B.POLICY_ALL)
    whole = step.out.clone()
    assert step.meta()["rows"] == 21 * 3 - 3 - 2 - 3
    assert step.pos[5].tolist() == [-1] * 3 and step.topk_idx[6].tolist() == [0, -1, -1] and int(step.step_meta[31]) == 8
    assert bool((whole[[5, 20]] == 0).all()) and bool((whole[6] != 0).any())
    step.out.fill_(7.0)
    step.eb_route(batch)
    step.eb_schedule(batch, 1, B.POLICY_ALL)
    step.eb_permute(batch)
    assert step.check_permutation(batch) == 0
    step.eb_expert_ffn_grouped()
    step.eb_combine(batch)
    assert torch.equal(step.out, whole)
    before = step.x.clone()
    step.eb_step(batch, 1, B.POLICY_ALL, in_place=True)
    assert torch.equal(step.x[5], before[5]) and not torch.equal(step.x[6], before[6])


@pytest.mark.parametrize("group_top", [1, 2])
@pytest.mark.parametrize("score", ["sigmoid", "softmax"])
def test_ties_go_to_the_lowest_index(score, group_top):
    E, K = 64, 6
    step, batch, layer_of = make(E, K, [50, 30])
    z = torch.round(normal((80, E), 3))               # a handful of values
    z[0], z[1] = 0.0, -0.0
    z[2] = torch.tensor([0.0, -0.0] * 32)
    bias = torch.round(2 * normal((3, E), 4)) / 4
    for b in (None, bias):
        for n_group, topk_group in ((1, 1), (8, 3), (16, 2)):
            check(step, batch, layer_of, z, B.Router(score, b, n_group, topk_group, group_top), b, 1)


@pytest.mark.parametrize("score", ["sigmoid", "softmax"])
def test_values_nearer_than_a_rounding_of_32_bits(score):
    """Biased scores that differ by 2^-24 to 2^-33 of their size, far less than 32-bit arithmetic tells apart: a bias makes up for the
    difference of two scores almost exactly."""
    E, K, T = 64, 6, 300
    step, batch, layer_of = make(E, K, [T], L=1)
    z = normal((1, E), 6).repeat(T, 1)                # every token the same logits but for its own small steps
    z += normal((T, E), 7, 2.0 ** -22)
    zd = z[0].double()
    s = torch.sigmoid(zd) if score == "sigmoid" else torch.softmax(zd, 0)
    bias = (1.0 - s).float().view(1, E)               # sums near 1
    check(step, batch, layer_of, z, B.Router(score, bias), bias, 1)
    check(step, batch, layer_of, z, B.Router(score, bias, 8, 3, 2), bias, 1)


@pytest.mark.parametrize("E", [8, 61, 256])
def test_types_and_strides(E):
    step, batch, layer_of = make(E, 4, [33, 65])
    wide = normal((98, E + 5), 4).to(torch.bfloat16)
    bias = normal((3, E), 5, 0.3)
    for z in (wide[:, 3:3 + E], wide[:, :E].contiguous(), wide.float()[:, 5:], wide.float()[:, 1:1 + E]):
        check(step, batch, layer_of, z, B.Router("sigmoid", bias), bias, 1)
        check(step, batch, layer_of, z, B.Router("softmax"), None, 1)


def test_as_the_contexts_router():
    """eb_route and whole steps gate by it until it is taken back; rows of micro-batches that are not routed stay."""
    step, batch, layer_of = make(16, 3, [20, 30, 11])
    z = normal((61, 16), 1)
    step.logits.copy_(z)
    bias = normal((3, 16), 2, 0.4)
    router = B.Router("sigmoid", bias, 4, 2, 2, scale=1.5)
    step.eb_route(batch)
    plain = step.topk_idx.clone()
    step.set_router(router)
    check(step, batch, layer_of, z, router, bias, 1, lambda: step.eb_route(batch))
    scored = step.topk_idx.clone()
    assert not torch.equal(scored, plain)
    step.topk_idx.fill_(77)
    step.eb_route(batch, 0b101)
    assert bool((step.topk_idx[20:50] == 77).all()) and torch.equal(step.topk_idx[:20], scored[:20]) and torch.equal(step.topk_idx[50:], scored[50:])
    step.eb_route_scored(batch, router, z, route_mask=0b010)
    assert torch.equal(step.topk_idx, scored)
    step.set_router(None)
    step.eb_route(batch)
    assert torch.equal(step.topk_idx, plain)


def test_many_tokens():
    """More blocks than fit the card at once, offsets beyond the first megabytes."""
    step, batch, _ = make(256, 8, [9000, 7000], D=8)
    z, bias = normal((16000, 256), 1), normal((3, 256), 2, 0.2)
    step.eb_route_scored(batch, B.Router("sigmoid", bias, 8, 4, 2), z)
    s = torch.sigmoid(z.double()) + torch.cat([bias[:1].double().expand(9000, -1), bias[1:2].double().expand(7000, -1)])
    best = s.view(-1, 8, 32).topk(2, dim=2).values.sum(2)
    kept = torch.zeros_like(best, dtype=torch.bool).scatter_(1, best.topk(4, dim=1).indices, True)
    want = torch.where(kept.repeat_interleave(32, 1), s, -1e9).topk(8, dim=1).indices
    assert torch.equal(step.topk_idx.long(), want)
