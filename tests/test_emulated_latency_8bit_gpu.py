"""The emulated expert-parallel latency loop times the expert pass that a step takes: that of the weights bound last."""
import itertools

import pytest
import torch

from paper_2608_07964_b200 import binding as B, driver, synth

pytestmark = pytest.mark.gpu


class Counted:
    """A step whose expert passes and dispatches are counted by name."""

    def __init__(self, step):
        self.calls = {}
        for name in ("eb_permute", "eb_permute_fp8", "eb_expert_ffn_grouped", "eb_expert_ffn_grouped_fp8"):
            setattr(step, name, self.counting(name, getattr(step, name)))

    def counting(self, name, call):
        def counted(*a, **k):
            self.calls[name] = self.calls.get(name, 0) + 1
            return call(*a, **k)
        return counted


@pytest.mark.parametrize("both", [False, True], ids=["8-bit", "8-bit last"])
def test_eight_bit_weights(both):
    wl = synth.workload("c1")
    step = B.from_workload(wl, fp8=True)
    w = [synth.all_weights(wl, k, "cuda") for k in ("gate", "up", "down")]
    q = list(itertools.chain(*[step.quantize_weights(t) for t in w]))
    if both:
        step.bind_weights(*w)
    step.bind_weights_fp8(*q)
    x0 = synth.packed_hidden(wl, device="cuda")
    logits_of = lambda j, l: synth.logits_for(wl, j, l, "cuda")  # noqa: E731
    counted = Counted(step)
    args = (step, wl.tok_off, wl.L, wl.D, wl.m, B.POLICY_MAXUTIL, logits_of, x0)
    r = driver.run_emulated_latency(*args)
    assert r["latency_ms"] > 0 and 0 < r["busy_ms"] <= wl.D * r["latency_ms"] * (1 + 1e-6)
    assert set(counted.calls) == {"eb_permute_fp8", "eb_expert_ffn_grouped_fp8"} and counted.calls["eb_permute_fp8"] == r["steps"]
    assert step.device_status() == 0
    if both:
        counted.calls.clear()
        step.bind_weights(*w)
        assert driver.run_emulated_latency(*args)["steps"] == r["steps"]
        assert set(counted.calls) == {"eb_permute", "eb_expert_ffn_grouped"}
