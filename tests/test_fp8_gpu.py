"""The 8-bit path against plain 64-bit forms: quantised weights and rows bit for bit, the grouped expert pass within a bound worked out
beforehand (reference64.ffn), whole steps against the calls one by one."""
import itertools

import numpy as np
import pytest
import torch

import reference64 as R64
from paper_2608_07964_b200 import binding as B, synth

pytestmark = pytest.mark.gpu
FP8 = torch.float8_e4m3fn


def normal(shape, seed, sigma=1.0, dtype=torch.bfloat16):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(shape, generator=gen, device="cuda") * sigma).to(dtype)


def bits(t):
    return t.contiguous().view(torch.uint8)


def any_step():
    return B.MoEStep(1, 1, 1, 0, 64, 64, 1, [0], 1)


# ---- weights ----------------------------------------------------------------------------------------
@pytest.mark.parametrize("shape", [(1, 1, 8), (1, 128, 128), (2, 129, 136), (3, 127, 120), (1, 300, 1000), (5, 1008, 720), (2, 3, 4, 40, 256)])
def test_quantized_weights_are_the_nearest_values(shape):
    w = normal(shape, 1, 0.02)
    flat = w.view(-1, *shape[-2:])
    flat[0, 0, :8] = 0.0
    if shape[-2] > 128:
        flat[-1, 128:, :128] = 0.0          # a block of zeros
    flat[0, :, -1] *= 64.0
    q, s = any_step().quantize_weights(w)
    assert q.shape == w.shape and s.shape == (*shape[:-2], -(-shape[-2] // 128), -(-shape[-1] // 128))
    for i, m in enumerate(flat):
        qr, sr = R64.quantise_weights(m.double())
        assert torch.equal(q.view(-1, *shape[-2:])[i].double(), qr)
        assert torch.equal(s.view(-1, *s.shape[-2:])[i], (sr * 448).float() / torch.full_like(sr, 448.0, dtype=torch.float32))


def test_quantized_halves_go_to_the_even_neighbour():
    """A maximum of 448 makes the scale 1: every bf16 value is rounded by itself, those between two e4m3 values to the even one."""
    grid = torch.arange(0, 127, dtype=torch.uint8, device="cuda").view(FP8).float()
    between = (grid[1:] + grid[:-1]) / 2                                   # at most 5 significant bits: bf16 has them
    row = torch.zeros(256, device="cuda")
    row[:127], row[127] = grid, 448.0
    row[128:128 + 126], row[255] = -between, 448.0
    q, s = any_step().quantize_weights(row.to(torch.bfloat16).view(1, 256).contiguous())
    assert torch.equal(s, torch.ones(1, 2, device="cuda"))
    assert torch.equal(q.double()[0], R64.nearest_e4m3(row.double()))
    # the same at maxima that are powers of two, very large and very small: 448 / m is no power of two then
    for m in (1.0, 2.0 ** 100, 2.0 ** -100, 2.0 ** 127, 2.0 ** -126, 2.0 ** -130):
        r = torch.cat([torch.arange(1, 257, device="cuda", dtype=torch.float64) / 256 * m]).to(torch.bfloat16)
        r[127], r[255] = m, m
        q, s = any_step().quantize_weights(r.view(1, 256).contiguous())
        assert torch.equal(q.double()[0], R64.nearest_e4m3(r.double() * 448 / m)), m
        assert torch.equal(s[0], torch.full((2,), m, device="cuda") / torch.full((2,), 448.0, device="cuda"))


def test_what_is_not_finite_makes_its_block_nan():
    w = normal((256, 256), 3)
    w[5, 130], w[200, 7] = float("inf"), float("nan")
    q, s = any_step().quantize_weights(w)
    assert torch.equal(torch.isnan(s), torch.tensor([[False, True], [True, False]], device="cuda"))
    ref, _ = R64.quantise_weights(w[:128, :128].double())
    assert torch.equal(q[:128, :128].double(), ref)


def test_no_weights_is_no_work():
    q, s = any_step().quantize_weights(torch.empty((0, 64, 64), dtype=torch.bfloat16, device="cuda"))
    assert q.numel() == 0 and s.shape == (0, 1, 1)


# ---- dispatch ---------------------------------------------------------------------------------------
SHAPES = [dict(L=2, E=4, K=2, S=0, H=16, I=16, D=2), dict(L=3, E=7, K=3, S=2, H=48, I=32, D=3), dict(L=2, E=8, K=2, S=1, H=128, I=64, D=4),
          dict(L=4, E=31, K=3, S=1, H=1008, I=720, D=5), dict(L=2, E=16, K=8, S=8, H=272, I=144, D=16), dict(L=3, E=64, K=6, S=2, H=2048, I=1408, D=8)]


def make(shape, tokens, layers=None, seed=0, capacity=0, **more):
    E, D = shape["E"], shape["D"]
    off = [0] + np.cumsum(tokens).tolist()
    step = B.MoEStep(shape["L"], E, shape["K"], shape["S"], shape["H"], shape["I"], D, [e * D // E for e in range(E)], max(off[-1], 1, capacity), fp8=True, **more)
    batch = B.Batch(off, [j % shape["L"] for j in range(len(tokens))] if layers is None else layers)
    T = off[-1]
    step.x[:T] = normal((T, shape["H"]), seed + 1)
    step.logits[:T] = normal((T, E), seed + 2, dtype=torch.float32)
    return step, batch, T


def weights8(step, seed):
    """Random weights, quantised by the library, bound; (gate, up, down) as ((q, scale) of matrix i) functions."""
    n, L, H, I = step.E + step.S, step.L, step.H, step.I
    w = [normal((L, n, I, H), seed, H ** -0.5), normal((L, n, I, H), seed + 1, H ** -0.5), normal((L, n, H, I), seed + 2, I ** -0.5)]
    qs = [step.quantize_weights(t) for t in w]
    step.bind_weights_fp8(*itertools.chain(*qs))
    return lambda i: [(q.view(-1, *q.shape[2:])[i], s.view(-1, *s.shape[2:])[i]) for q, s in qs]


@pytest.mark.parametrize("tokens", [[1], [5, 0, 9], [32, 33], [300, 7, 61], [400, 380, 390], [1500, 1100]])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: f"E{s['E']}H{s['H']}")
def test_dispatch_quantises_the_rows_of_the_plain_one(shape, tokens):
    """The tables are those of eb_permute, a row is its token's row quantised; by the calls and inside a step."""
    step, batch, T = make(shape, tokens)
    if T > 8:
        step.x[1] = 0.0
        step.x[3, :8] *= 1e30
        step.x[4] *= 1e-30
    step.eb_route(batch)
    step.eb_schedule(batch, 1, B.POLICY_ALL)
    step.eb_permute(batch)
    R, G = step.meta()["rows"], step.meta()["groups"]
    tables = lambda: [t.clone() for t in (step.group_off[:G + 1], step.group_w[:G], step.row_src[:R], step.pos[:T], step.step_meta)]  # noqa: E731
    plain = tables()
    q, s = R64.quantise_rows(step.x[:T].double())
    src = step.row_src[:R].long()
    s32 = (s * 448).float() / torch.full(s.shape, 448.0, device="cuda")
    by_calls = None
    for whole in (False, True):
        step.xp.view(torch.uint8).fill_(0xA5)
        if whole:
            weights8(step, 5)
            step.eb_step(batch, 1, B.POLICY_ALL)
        else:
            step.eb_permute_fp8(batch)
        for a, b in zip(plain, tables()):
            assert torch.equal(a, b)
        assert torch.equal(step.xq[:R].double(), q[src])
        assert torch.equal(step.xs[:R], s32[src])
        if R < step.rows_cap:
            assert bool((bits(step.xq[R:]) == 0xA5).all()) and bool((bits(step.xs[R:]) == 0xA5).all())
        now = bits(step.xq[:R]).clone()
        assert by_calls is None or torch.equal(by_calls, now)
        by_calls = now
    assert step.device_status() == 0


# ---- expert pass ------------------------------------------------------------------------------------
def table_of(step, sizes):
    """The group table of one layer and one device whose experts have these numbers of rows."""
    G, R = len(sizes), sum(sizes)
    step.group_off[:G + 1] = torch.tensor([0] + np.cumsum(sizes).tolist(), dtype=torch.int32)
    step.group_w[:G] = torch.arange(G, dtype=torch.int32)
    step.step_meta[:5] = torch.tensor([R, G, 1, 0, G], dtype=torch.int32)
    return R


def within(y, ref, tol):
    off = (y.double() - ref).abs()
    assert bool((off <= tol).all()), f"{float((off / tol).max()):.3g} of the bound at {int((off / tol).argmax())}"


def check_groups(step, get, n_groups=None):
    """yp against the plain form, group by group."""
    m = step.meta()
    off, gw = step.group_off[:m["groups"] + 1].tolist(), step.group_w[:m["groups"]].tolist()
    for g in range(m["groups"] if n_groups is None else n_groups):
        if off[g + 1] > off[g]:
            rows = slice(off[g], off[g + 1])
            within(step.yp[rows], *R64.ffn(step.xq[rows], step.xs[rows], *get(gw[g])))


def fill_rows(step, R, seed):
    q, s = R64.quantise_rows(normal((R, step.H), seed).double())
    step.xq[:R], step.xs[:R] = q.float().to(FP8), s.float()


SIZES = [[1], [0, 3, 0, 17], [16, 15, 32, 31], [33, 64, 65, 1], [100, 128, 129, 0], [256, 257, 300, 96], [700, 5, 48, 112]]


def expert_step(sizes, H, I, many):
    """A context of one layer and one device for groups of these sizes, whose capacity chooses the kernel for few or for many rows an expert."""
    R, E = sum(sizes), len(sizes)
    if many:
        return B.MoEStep(1, E, 1, 0, H, I, 1, [0] * E, max(R + 3, 64 * E + 1), fp8=True)
    E = max(E, -(-(R + 3) // 64))
    return B.MoEStep(1, E, 1, 0, H, I, 1, [0] * E, R + 3, fp8=True)


@pytest.mark.parametrize("many", [False, True], ids=["few", "many"])
@pytest.mark.parametrize("sizes", SIZES, ids=str)
@pytest.mark.parametrize("H,I", [(16, 16), (128, 128), (144, 272), (512, 256), (1008, 720), (2048, 1408), (640, 4112)])
def test_expert_pass(H, I, sizes, many):
    R = sum(sizes)
    step = expert_step(sizes, H, I, many)
    get = weights8(step, H + I)
    assert table_of(step, sizes) == R
    fill_rows(step, R, 7)
    bits(step.xq[R:]).fill_(0x7F)            # rows behind the last one: NaN values, never stored
    step.xs[R:] = float("nan")
    step.yp.fill_(-3.0)
    step.eb_expert_ffn_grouped_fp8()
    assert step.device_status() == 0 and step.check_workspace_guards() == 0
    check_groups(step, get)
    assert bool((step.yp[R:] == -3.0).all())
    first = step.yp[:R].clone()
    for _ in range(3):
        step.yp.zero_()
        step.eb_expert_ffn_grouped_fp8()
        assert torch.equal(step.yp[:R], first)          # whatever the order of the tiles


@pytest.mark.parametrize("most", [128, 1000])   # rows of the context: the kernel for few rows an expert, for many
def test_scales_that_differ_from_block_to_block(most):
    """Scales over many powers of two: a block whose scale were taken for another's would stand out."""
    H, I, sizes = 1024, 640, [40, 88] if most == 128 else [40, 200]
    step = B.MoEStep(1, 2, 1, 0, H, I, 1, [0, 0], most, fp8=True)
    gen = torch.Generator(device="cuda").manual_seed(11)
    e4m3 = lambda *s: (torch.randn(s, generator=gen, device="cuda") * 100).clamp(-448, 448).to(FP8)  # noqa: E731
    wide = lambda mid, *s: mid * torch.exp2(8 * torch.rand(s, generator=gen, device="cuda") - 4)      # noqa: E731
    w = [(e4m3(1, 2, I, H), wide(2e-5, 1, 2, 5, 8)), (e4m3(1, 2, I, H), wide(2e-5, 1, 2, 5, 8)), (e4m3(1, 2, H, I), wide(2e-4, 1, 2, 8, 5))]
    step.bind_weights_fp8(*itertools.chain(*w))
    R = table_of(step, sizes)
    step.xq[:R], step.xs[:R] = e4m3(R, H), wide(0.01, R, 8)
    step.eb_expert_ffn_grouped_fp8()
    check_groups(step, lambda i: [(q[0, i], s[0, i]) for q, s in w])


@pytest.mark.parametrize("most", [128, 1000])
def test_zeros_and_what_is_not_finite(most):
    H, I, sizes = 256, 384, [6, 70]
    step = B.MoEStep(1, 2, 1, 0, H, I, 1, [0, 0], most, fp8=True)
    get = weights8(step, 2)
    R = table_of(step, sizes)
    fill_rows(step, R, 3)
    step.xs[0] = 0.0                          # a token of zeros
    step.xs[2, 1] = float("nan")              # as eb_permute_fp8 marks a block with an infinity
    step.xs[50, 0] = float("inf")
    step.eb_expert_ffn_grouped_fp8()
    assert bool((step.yp[0] == 0).all())
    bad = torch.zeros(R, dtype=torch.bool, device="cuda")
    bad[[2, 50]] = True
    assert torch.equal(torch.isnan(step.yp[:R].float()).all(1), bad) and torch.equal(torch.isnan(step.yp[:R].float()).any(1), bad)
    good = torch.nonzero(~bad[6:]).flatten() + 6
    within(step.yp[good], *R64.ffn(step.xq[good], step.xs[good], *get(1)))


@pytest.mark.parametrize("capacity", [0, 1 << 12], ids=["few", "many"])
@pytest.mark.parametrize("tokens", [[1, 1, 1], [4, 30, 9], [64, 64], [150, 500, 31]])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: f"E{s['E']}H{s['H']}")
def test_steps_with_shared_experts_and_a_router(shape, tokens, capacity):
    """Router, schedule, quantising dispatch, expert pass and aggregation as they are used together: by the calls one by one against the
    plain forms, then as whole steps, in place, from a graph and on another stream, bit for bit."""
    step, batch, T = make(shape, tokens, capacity=capacity)
    get = weights8(step, 9)
    bias = 0.3 * normal((shape["L"], shape["E"]), 4, dtype=torch.float32)
    router = B.Router("sigmoid", bias, scale=2.0)
    step.eb_route_scored(batch, router)
    step.eb_schedule(batch, 1, B.POLICY_ALL)
    step.eb_permute_fp8(batch)
    assert step.check_permutation(batch) == 0
    step.eb_expert_ffn_grouped_fp8()
    step.eb_combine(batch)
    assert step.device_status() == 0 and step.check_workspace_guards() == 0
    m = step.meta()
    check_groups(step, get)
    # aggregation of what the pass gave, in 64 bits: K + S products, one rounding to bf16
    w = torch.cat([step.topk_w[:T].double(), torch.ones((T, step.S), dtype=torch.float64, device="cuda")], 1)
    rows = step.yp.double()[step.pos[:T].long()]
    out = (w[..., None] * rows).sum(1)
    tol = 2.0 ** -8 * out.abs() + 20 * 2.0 ** -24 * (w[..., None] * rows).abs().sum(1) + 1e-30
    within(step.out[:T], out, tol)
    want, idx, yp = step.out[:T].clone(), step.topk_idx[:T].clone(), step.yp[:m["rows"]].clone()

    step.set_router(router)
    step.out.zero_(), step.yp.zero_(), step.topk_idx.zero_()
    step.eb_step(batch, 1, B.POLICY_ALL)
    assert torch.equal(step.topk_idx[:T], idx) and torch.equal(step.out[:T], want) and torch.equal(step.yp[:m["rows"]], yp)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step.eb_step(batch, 1, B.POLICY_ALL)
    step.set_router(None)                      # the graph keeps its router
    for _ in range(2):
        step.out.zero_(), step.topk_idx.zero_()
        graph.replay()
        assert torch.equal(step.topk_idx[:T], idx) and torch.equal(step.out[:T], want)
    step.set_router(router)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step.out.zero_()
        step.eb_step(batch, 1, B.POLICY_ALL)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(step.out[:T], want)
    before = step.x[:T].clone()
    step.eb_step(batch, 1, B.POLICY_ALL, in_place=True)
    out2 = out + before.double()
    within(step.x[:T], out2, 2.0 ** -8 * out2.abs() + tol)


def test_both_kinds_of_weights_may_be_bound():
    """The step takes those bound last; the calls by name take theirs; a device's share is the whole pass's rows."""
    shape = SHAPES[2]
    step, batch, T = make(shape, [40, 25])
    wl = [normal((2, 9, 64, 128), 1, 0.1), normal((2, 9, 64, 128), 2, 0.1), normal((2, 9, 128, 64), 3, 0.1)]
    step.bind_weights(*wl)
    step.eb_step(batch, 1, B.POLICY_ALL)
    plain = step.out[:T].clone()
    weights8(step, 5)
    step.eb_step(batch, 1, B.POLICY_ALL)
    eight = step.out[:T].clone()
    assert not torch.equal(plain, eight)
    step.eb_permute(batch)
    step.eb_expert_ffn_grouped()
    step.eb_combine(batch)
    assert torch.equal(step.out[:T], plain)
    step.eb_permute_fp8(batch)
    step.eb_expert_ffn_grouped_fp8()
    step.eb_combine(batch)
    assert torch.equal(step.out[:T], eight)
    whole = step.yp.clone()
    for timed in (False, True):
        step.set_timing(timed)
        step.yp.zero_()
        for d in range(step.D):
            step.eb_expert_ffn_grouped_fp8(device=d)
        R = step.meta()["rows"]
        assert torch.equal(step.yp[:R], whole[:R])
    assert step.kernel_ms()["ffn_gateup"] > 0
    step.set_timing(False)
    step.bind_weights(*wl)
    step.eb_step(batch, 1, B.POLICY_ALL)
    assert torch.equal(step.out[:T], plain)


def test_deferred_micro_batches_are_left_alone():
    shape = SHAPES[1]
    step, batch, T = make(shape, [9, 14, 20, 6])
    weights8(step, 5)
    step.out.fill_(5.0)
    step.eb_step(batch, 2, B.POLICY_MAXUTIL)
    run = step.sched_result()["run_mask"]
    for j in range(4):
        rows = step.out[batch.tok_off[j]:batch.tok_off[j + 1]]
        assert bool((rows == 5.0).all()) != bool((run >> j) & 1)
    assert step.check_permutation(batch) == 0


@pytest.mark.parametrize("capacity", [0, 1 << 12], ids=["few", "many"])
def test_two_contexts_and_streams_at_once(capacity):
    """Contexts of their own on streams of their own: what they compute does not depend on each other."""
    shape = SHAPES[3]
    made = [make(shape, [60, 33, 90], seed=k, capacity=capacity) for k in (0, 10)]
    streams, want = [torch.cuda.Stream() for _ in made], []
    for step, batch, T in made:
        weights8(step, 9)
        step.eb_step(batch, 1, B.POLICY_ALL)
        want.append(step.out[:T].clone())
    torch.cuda.synchronize()
    for _ in range(20):
        for (step, batch, T), s in zip(made, streams):
            with torch.cuda.stream(s):
                step.eb_step(batch, 1, B.POLICY_ALL)
    torch.cuda.synchronize()
    for (step, batch, T), w in zip(made, want):
        assert torch.equal(step.out[:T], w) and step.device_status() == 0 and step.check_workspace_guards() == 0


def test_host_steps_and_runs_use_the_weights_bound_last():
    from paper_2608_07964_b200 import driver
    wl = synth.workload("c1")
    step = B.from_workload(wl, fp8=True)
    T = wl.T_tot
    w = [synth.all_weights(wl, k, "cuda") for k in ("gate", "up", "down")]
    step.bind_weights_fp8(*itertools.chain(*[step.quantize_weights(t) for t in w]))
    step.set_router(B.Router("sigmoid", n_group=4, topk_group=2, group_top=2))
    lg, x = synth.packed_logits(wl), synth.packed_hidden(wl)
    batch = B.Batch(wl.tok_off, wl.layers)
    h_out = torch.zeros((T, wl.H), dtype=torch.bfloat16).pin_memory()
    step.out.zero_()                          # rows of the deferred micro-batch are left as they are, and compared too
    res = step.eb_step_host(batch, wl.m, lg.pin_memory(), x.pin_memory(), h_out)
    step.logits[:T], step.x[:T] = lg.cuda(), x.cuda()
    step.eb_step(batch, wl.m)
    assert step.sched_result()["run_mask"] == res["run_mask"]
    assert torch.equal(step.out[:T].cpu(), h_out)
    logits_of = lambda j, l: synth.logits_for(wl, j, l, "cuda")  # noqa: E731
    x0 = 0.05 * synth.packed_hidden(wl, device="cuda")
    a = driver.run_full(step, wl.tok_off, wl.L, wl.m, B.POLICY_MAXUTIL, logits_of, x0)
    g = driver.StepGraphs(step, wl.tok_off)
    b = driver.run_full(step, wl.tok_off, wl.L, wl.m, B.POLICY_MAXUTIL, logits_of, x0, graphs=g)
    assert torch.equal(a["x"], b["x"]) and bool(torch.isfinite(a["x"].float()).all())
