"""What the host code of the router with scores and of the 8-bit path refuses and launches, on the CPU, against the stand-in runtime."""
import ctypes as C

import pytest

from paper_2608_07964_b200 import binding as B
from test_launch_chain import EB_ERR_CUDA, Context, lib  # noqa: F401  (the fixture)

INVALID, UNSUPPORTED, WORKSPACE = 1, 2, 3
P = 1 << 30


def context(lib, fp8=True, tokens=4096, **more):
    c = Context(lib, **{**dict(E=8, K=2, S=1, D=4, max_tokens=tokens), **more})
    if fp8:
        assert lib.eb_enable_fp8(c.ctx) == 0
        assert lib.eb_set_workspace(c.ctx, 1 << 20, lib.eb_workspace_bytes(c.ctx)) == 0
        assert lib.eb_bind_weights_fp8(c.ctx, P, P, P, P, P, P) == 0
    return c


def router(score=1, n_group=4, topk_group=2, group_top=2, scale=1.0, bias=None):
    return B.EbRouter(score, n_group, topk_group, group_top, scale, bias)


BAD = [dict(score=2), dict(score=-1), dict(n_group=0), dict(n_group=3), dict(n_group=64), dict(topk_group=0), dict(topk_group=5), dict(group_top=0),
       dict(group_top=3), dict(n_group=8, topk_group=1), dict(scale=0.0), dict(scale=-1.0), dict(scale=float("nan")), dict(scale=float("inf")), dict(bias=P + 2)]


@pytest.mark.parametrize("bad", BAD, ids=str)
def test_routers_that_make_no_sense(lib, bad):
    lib.fake_reset(-1)
    c = context(lib, fp8=False)
    b, r = c.batch(3, 5), router(**bad)
    assert lib.eb_route_scored(c.ctx, None, C.byref(b.c), 7, C.byref(r), P, 0, 8, P, P, P, P) == INVALID
    assert lib.eb_set_router(c.ctx, C.byref(r)) == INVALID
    assert lib.eb_last_error(c.ctx) and c.names() == []


def test_logits_and_masks_of_the_router(lib):
    lib.fake_reset(-1)
    c = context(lib, fp8=False)
    b, r = c.batch(3, 5), router()
    call = lambda logits=P, kind=0, stride=8, mask=7, rr=C.byref(r), out=P: lib.eb_route_scored(  # noqa: E731
        c.ctx, None, C.byref(b.c), mask, rr, logits, kind, stride, out, P, P, P)
    assert call(kind=2) == UNSUPPORTED and call(stride=7) == INVALID and call(logits=None) == INVALID and call(out=None) == INVALID
    assert call(logits=P + 2) == INVALID and call(logits=P + 1, kind=1) == INVALID and call(mask=8) == INVALID and call(rr=None) == INVALID
    assert lib.eb_route_scored(None, None, C.byref(b.c), 7, C.byref(r), P, 0, 8, P, P, P, P) == INVALID
    assert lib.eb_set_router(None, None) == INVALID
    assert c.names() == []
    assert call(mask=0) == 0 and c.names() == []
    assert call(logits=P + 2, kind=1, stride=9) == 0 and len(c.names()) == 2
    empty = c.batch(0, 0)
    assert lib.eb_route_scored(c.ctx, None, C.byref(empty.c), 0, C.byref(r), P, 0, 8, P, P, P, P) == 0


def test_the_router_of_a_context_stays_until_it_is_taken_back(lib):
    lib.fake_reset(-1)
    c = context(lib, fp8=False)
    plain = c.step(3, 5) == 0 and c.names()
    r = router()
    assert lib.eb_set_router(c.ctx, C.byref(r)) == 0
    assert lib.eb_set_router(c.ctx, C.byref(router(score=9))) == INVALID      # refused: the first one stays
    lib.fake_reset(-1)
    assert c.step(3, 5) == 0 and c.names() != plain
    scored = c.names()
    lib.fake_reset(-1)
    assert c.step(3, 5) == 0 and c.names() == scored
    assert lib.eb_set_router(c.ctx, None) == 0
    lib.fake_reset(-1)
    assert c.step(3, 5) == 0 and c.names() == plain


def test_eight_bit_calls_need_a_context_laid_out_for_them(lib):
    lib.fake_reset(-1)
    c = context(lib, fp8=False)
    b = c.batch(3, 5)
    assert lib.eb_bind_weights_fp8(c.ctx, P, P, P, P, P, P) == INVALID
    assert lib.eb_permute_fp8(c.ctx, None, C.byref(b.c), P, P, P, P, P, P, P, P, P, P) == INVALID
    assert lib.eb_expert_ffn_grouped_fp8(c.ctx, None, P, P, P, P, P, P, -1) == INVALID
    before = lib.eb_workspace_bytes(c.ctx)
    assert lib.eb_enable_fp8(c.ctx) == 0 and lib.eb_enable_fp8(c.ctx) == 0
    assert lib.eb_workspace_bytes(c.ctx) > before
    assert c.step(3, 5) == WORKSPACE                                          # the old one is too small now
    assert lib.eb_set_workspace(c.ctx, 1 << 20, before) == WORKSPACE
    assert lib.eb_set_workspace(c.ctx, 1 << 20, lib.eb_workspace_bytes(c.ctx)) == 0
    assert c.step(3, 5) == 0                                                  # bf16 weights are bound
    assert lib.eb_expert_ffn_grouped_fp8(c.ctx, None, P, P, P, P, P, P, -1) == INVALID
    for sizes in (dict(H=72), dict(I=40)):
        odd = context(lib, fp8=False, **sizes)
        assert lib.eb_enable_fp8(odd.ctx) == UNSUPPORTED
    assert lib.eb_enable_fp8(None) == INVALID


def test_eight_bit_arguments(lib):
    lib.fake_reset(-1)
    c = context(lib)
    b = c.batch(3, 5)
    for i in range(6):
        for wrong in (None, P + 8):
            args = [P] * 6
            args[i] = wrong
            assert lib.eb_bind_weights_fp8(c.ctx, *args) == INVALID, i
    for i in range(10):
        args = [P] * 10
        args[i] = None
        assert lib.eb_permute_fp8(c.ctx, None, C.byref(b.c), *args) == INVALID, i
    for i in range(6):
        args = [P] * 6
        args[i] = None
        assert lib.eb_expert_ffn_grouped_fp8(c.ctx, None, *args, -1) == INVALID, i
    assert lib.eb_permute_fp8(c.ctx, None, C.byref(b.c), P, P, P, P, P, P, P, P + 8, P, P) == INVALID
    assert lib.eb_permute_fp8(c.ctx, None, C.byref(b.c), P, P, P, P, P, P, P, P, P + 4, P) == INVALID
    assert lib.eb_expert_ffn_grouped_fp8(c.ctx, None, P + 8, P, P, P, P, P, -1) == INVALID
    assert lib.eb_expert_ffn_grouped_fp8(c.ctx, None, P, P, P, P, P, P, 4) == INVALID
    q = lambda w=P, n=2, rows=3, cols=16, to=P, s=P: lib.eb_quantize_weights(c.ctx, None, w, n, rows, cols, to, s)  # noqa: E731
    assert q(w=None) == INVALID and q(to=None) == INVALID and q(s=None) == INVALID and q(w=P + 8) == INVALID and q(to=P + 8) == INVALID and q(s=P + 2) == INVALID
    assert q(n=-1) == INVALID and q(rows=-1) == INVALID and q(cols=-8) == INVALID and q(cols=12) == UNSUPPORTED
    assert q(n=0) == 0 and q(rows=0) == 0 and q(cols=0, w=None) == 0
    assert c.names() == []
    assert q(n=70000) == 0 and len(c.names()) == 2                            # 65535 matrices a launch


def test_capacity_chooses_the_kernel(lib):
    """At most 64 rows an expert on average, the largest batch at one layer: by tiles of 128 rows."""
    for tokens, name in ((256, "ffn8_few_kernel"), (257, "ffn8_many_kernel")):   # E = 8, K = 2
        lib.fake_reset(-1)
        c = context(lib, tokens=tokens)
        assert c.step(3, 5) == 0
        assert sum(name in n for n in c.names()) == 1, c.names()


@pytest.mark.parametrize("timing", [0, 1])
@pytest.mark.parametrize("tokens", [256, 4096])
def test_nothing_is_launched_behind_a_refused_kernel(lib, tokens, timing):
    lib.fake_reset(-1)
    c = context(lib, tokens=tokens)
    assert lib.eb_set_timing(c.ctx, timing) == 0
    b, r = c.batch(3, 5), router()
    calls = dict(route=lambda: lib.eb_route_scored(c.ctx, None, C.byref(b.c), 7, C.byref(r), P, 0, 8, P, P, P, P),
                 quantize=lambda: lib.eb_quantize_weights(c.ctx, None, P, 3, 40, 48, P, P),
                 permute=lambda: lib.eb_permute_fp8(c.ctx, None, C.byref(b.c), P, P, P, P, P, P, P, P, P, P),
                 experts=lambda: lib.eb_expert_ffn_grouped_fp8(c.ctx, None, P, P, P, P, P, P, -1),
                 device=lambda: lib.eb_expert_ffn_grouped_fp8(c.ctx, None, P, P, P, P, P, P, 1),
                 step=lambda: c.step(3, 5))
    for name, call in calls.items():
        lib.fake_reset(-1)
        assert call() == 0, name
        chain = c.names()
        assert chain, name
        for i in range(len(chain)):
            lib.fake_reset(i)
            assert call() == EB_ERR_CUDA, (name, chain[i])
            assert c.names() == chain[:i], (name, chain[i])
        lib.fake_reset(-1)
        assert call() == 0 and c.names() == chain, name
