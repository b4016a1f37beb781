"""The 8-bit expert pass where gates are far below zero: silu(g) = g / (1 + e^-g) falls to nothing there, and a block of such values is
stored by its own largest magnitude, so each has to be right to its own size."""
import pytest
import torch

import reference64 as R64
from paper_2608_07964_b200 import binding as B
from test_fp8_gpu import bits, expert_step, table_of, within

pytestmark = pytest.mark.gpu
FP8 = torch.float8_e4m3fn
H, I = 256, 512


def pass_and_bound(step, R, gate, up, down, s_up):
    """What the pass should give for rows whose gate and up sums are exact in 32 bits (few terms, scales that are powers of two), and a bound.

    Then silu(g) u is off by its own arithmetic alone: e^-|g| by way of a power of two whose argument, |g| log2 e rounded twice, is off by
    |g| 2^-22 at most, 2^-22 for the power, and five roundings and a reciprocal (2^-23): (|g| + 8) 2^-22 of its size.  Rounded to e4m3 with the
    block's largest magnitude, which is as far off, an interval that holds a rounding border may end at either side of it."""
    x = step.xq[:R].double() * R64.spread(step.xs[:R].double(), 1)[:, :H]
    g, u = x @ gate.double().T, x @ up.double().T * s_up
    h = g * torch.exp(-torch.nn.functional.softplus(-g)) * u            # sigmoid(g) = exp(-log(1 + e^-g)), right down to its smallest values
    rel = (g.abs() + 8) * 2.0 ** -22
    hb, rb = h.view(R, -1, 128), rel.view(R, -1, 128)
    m = hb.abs().amax(2, keepdim=True)
    none = m < 2.0 ** -110                                              # counts as zeros
    unit = torch.where(none, 0.0, R64.TOP / m.clamp_min(1e-300))
    off = hb.abs() * (rb + rb.amax(2, keepdim=True))
    q = R64.nearest_e4m3(hb * unit)
    lo, hi = (R64.nearest_e4m3(((hb + k * off) * unit).clamp(-R64.TOP, R64.TOP)) for k in (-1, 1))
    back = torch.where(none, 0.0, m / R64.TOP)
    a = (q * back).view(R, I)
    da = ((hi - lo) * back).view(R, I) + a.abs() * rb.amax(2, keepdim=True).expand_as(hb).reshape(R, I)
    wd = down.double()
    y = a @ wd.T
    tol = da @ wd.abs().T + 2 * (I + 8) * 2.0 ** -24 * (a.abs() @ wd.abs().T)
    return y, tol + 2.0 ** -8 * (y.abs() + tol) + 2.0 ** -126


def run(many, gate_of_block, s_up=1.0, rows=6):
    """Rows of three ones (and multiples of a half for up) against gate weights whose sums are `gate_of_block` of each block of 128 outputs, less up to 2."""
    sizes = [rows, 37]
    step = expert_step(sizes, H, I, many)
    R = table_of(step, sizes)
    E = step.E
    gen = torch.Generator(device="cuda").manual_seed(5)
    gate, up = torch.zeros((I, H), device="cuda"), torch.zeros((I, H), device="cuda")
    for b, g in enumerate(gate_of_block):
        gate[128 * b:128 * b + 128, 0] = g
    gate[:, 1] = -torch.randint(0, 9, (I,), generator=gen, device="cuda") / 4.0      # sums of a whole number and of quarters
    up[:, 2] = torch.randint(-14, 15, (I,), generator=gen, device="cuda") / 8.0
    up[:, 2][up[:, 2] == 0] = 1.0
    down = torch.randn((H, I), generator=gen, device="cuda").clamp(-3, 3).to(FP8).float()
    for t in (gate, up):
        assert torch.equal(t.to(FP8).float(), t)
    ones = lambda *s: torch.ones((1, E, *s), device="cuda")  # noqa: E731
    w8 = lambda t: t.to(FP8).expand(1, E, *t.shape).contiguous()  # noqa: E731
    step.bind_weights_fp8(w8(gate), ones(I // 128, H // 128), w8(up), s_up * ones(I // 128, H // 128), w8(down), ones(H // 128, I // 128))
    x = torch.zeros((R, H), device="cuda")
    x[:, 0] = 1.0
    x[:, 1] = 1.0
    x[:, 2] = 0.5 * (1 + torch.arange(R, device="cuda") % 4)
    step.xq[:R], step.xs[:R] = x.to(FP8), 1.0
    bits(step.xq[R:]).fill_(0x7F)
    step.yp.fill_(-3.0)
    step.eb_expert_ffn_grouped_fp8()
    assert step.device_status() == 0
    return step, R, pass_and_bound(step, R, gate, up, down, s_up)


@pytest.mark.parametrize("gates", [[-36, -40, -44, -48], [-44, -44, -44, -44], [-60, -60, -60, -60], [-72, -72, -72, -72], [-60, 4, -72, -20], [0, -1, 2, 8]], ids=str)
@pytest.mark.parametrize("many", [False, True], ids=["few", "many"])
def test_blocks_of_far_gates(many, gates):
    step, R, (y, tol) = run(many, gates)
    within(step.yp[:R], y, tol)


@pytest.mark.parametrize("many", [False, True], ids=["few", "many"])
def test_gates_whose_sigmoid_vanishes(many):
    """e^-104 and below: no 32-bit number is that small, and neither is anything made from it."""
    step, R, (y, tol) = run(many, [-104, -112, -240, -448])
    assert bool((step.yp[:R] == 0).all())


@pytest.mark.parametrize("many", [False, True], ids=["few", "many"])
def test_a_gate_and_an_output_whose_product_is_too_large(many):
    """g u is beyond 32 bits, silu(g) u is not."""
    step, R, (y, tol) = run(many, [-44, -60, -72, -52], s_up=2.0 ** 125)
    assert bool(torch.isfinite(y).all()) and float(y.abs().max()) > 1e6
    within(step.yp[:R], y, tol)


@pytest.mark.parametrize("many", [False, True], ids=["few", "many"])
def test_a_gate_that_is_not_a_number_stays_with_its_row(many):
    sizes = [20, 37]
    step = expert_step(sizes, H, I, many)
    R = table_of(step, sizes)
    E = step.E
    w = lambda *s: torch.full((1, E, *s), 0.5, device="cuda").to(FP8)  # noqa: E731
    one = lambda *s: torch.ones((1, E, *s), device="cuda")  # noqa: E731
    step.bind_weights_fp8(w(I, H), one(4, 2), w(I, H), one(4, 2), w(H, I), one(2, 4))
    step.xq[:R], step.xs[:R] = torch.full((R, H), 0.25, device="cuda").to(FP8), 2.0 ** -6
    step.xs[3], step.xs[30] = float("nan"), float("-inf")
    step.eb_expert_ffn_grouped_fp8()
    bad = torch.zeros(R, dtype=torch.bool, device="cuda")
    bad[[3, 30]] = True
    y = step.yp[:R].float()
    assert torch.equal(torch.isnan(y).all(1), bad) and torch.equal(torch.isnan(y).any(1), bad)
