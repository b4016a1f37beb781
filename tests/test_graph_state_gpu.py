"""Steps replayed from graphs follow the router and the weights of the context: what is set or bound between two runs holds for the second."""
import itertools

import pytest
import torch

from paper_2608_07964_b200 import binding as B, driver, synth

pytestmark = pytest.mark.gpu


class Runs:
    """The same run of Algorithm 1 with and without graphs."""

    def __init__(self):
        self.wl = wl = synth.workload("c1")
        self.step = B.from_workload(wl, fp8=True)
        self.w = [synth.all_weights(wl, k, "cuda") for k in ("gate", "up", "down")]
        self.q = list(itertools.chain(*[self.step.quantize_weights(t) for t in self.w]))
        self.x0 = 0.05 * synth.packed_hidden(wl, device="cuda")
        self.graphs = driver.StepGraphs(self.step, wl.tok_off)
        self.bias = [0.4 * torch.randn((wl.L, wl.E), generator=torch.Generator(device="cuda").manual_seed(k), device="cuda") for k in (1, 2)]

    def run(self, graphs):
        wl = self.wl
        logits_of = lambda j, l: synth.logits_for(wl, j, l, "cuda")  # noqa: E731
        r = driver.run_full(self.step, wl.tok_off, wl.L, wl.m, B.POLICY_MAXUTIL, logits_of, self.x0, graphs=graphs)
        return r["x"], r["steps"]

    def same(self):
        """Both runs agree; the hidden states, and how many steps were captured."""
        x, steps = self.run(None)
        before = self.graphs.captures
        gx, gsteps = self.run(self.graphs)
        assert gsteps == steps and torch.equal(gx, x)
        made = self.graphs.captures - before
        again, _ = self.run(self.graphs)
        assert torch.equal(again, x) and self.graphs.captures == before + made      # nothing changed: all of it replayed
        return x, made


def test_a_router_set_between_two_runs():
    r = Runs()
    r.step.bind_weights(*r.w)
    routers = [None, B.Router("sigmoid", r.bias[0], 4, 2, 2), B.Router("sigmoid", r.bias[1], 4, 2, 2), B.Router("softmax", scale=0.5), None]
    seen = []
    for router in routers:
        r.step.set_router(router)
        x, made = r.same()
        assert made > 0
        seen.append(x)
    assert torch.equal(seen[0], seen[-1])
    assert not any(torch.equal(a, b) for a, b in itertools.combinations(seen[:-1], 2))


def test_weights_bound_between_two_runs():
    r = Runs()
    other = [(0.5 * t.float()).to(torch.bfloat16) for t in r.w]
    seen = []
    for bind in (lambda: r.step.bind_weights(*r.w), lambda: r.step.bind_weights_fp8(*r.q), lambda: r.step.bind_weights(*other),
                 lambda: r.step.bind_weights(*r.w)):
        bind()
        x, made = r.same()
        assert made > 0
        seen.append(x)
    assert torch.equal(seen[0], seen[-1])
    assert not any(torch.equal(a, b) for a, b in itertools.combinations(seen[:-1], 2))


def test_graphs_of_an_earlier_state_are_let_go():
    r = Runs()
    r.step.bind_weights(*r.w)
    _, made = r.same()
    assert len(r.graphs.graphs) == made
    r.step.set_router(B.Router("sigmoid", r.bias[0]))
    _, made = r.same()
    assert len(r.graphs.graphs) == made
