"""Rates at and below zero of the AdamW step, as a number and on the device (GPU)."""
import math

import numpy as np
import pytest
import torch

from paper_2412_07210_amd import EditOuterError
from test_gpu_adamw import DEV, Run

pytestmark = pytest.mark.gpu

KINDS = [("f32", "f32", False), ("bf16", "e4m3", True)]
# few blocks decide in the update pass, many or with a tensor left out before it
MISSING = [(), (1,)]


def on_device(x):
    return torch.full((1,), x, dtype=torch.float64, device=DEV)


@pytest.mark.parametrize("missing", MISSING, ids=["fused", "apart"])
@pytest.mark.parametrize("dtype,state,stochastic", KINDS)
def test_a_rate_of_either_zero_moves_no_parameter(dtype, state, stochastic, missing):
    """m is not 0, and decays and gradients still reach the states: t goes on."""
    run = Run([700, 300, 5000], dtype, None, state, seed=21, no_grad=missing, stochastic=stochastic)
    run.step(lr=1e-3)
    for t, lr in enumerate((0.0, -0.0, on_device(0.0), on_device(-0.0))):
        run.draw(t + 1)
        keep = run.flat_p.clone()
        run.step(lr=lr, max_norm=0.5 if t % 2 else None, seed=t)
        assert torch.equal(run.flat_p, keep), (t, lr)
    run.draw(9)
    run.step(lr=1e-3)
    assert run.opt.state_get().step == 6
    run.close()


@pytest.mark.parametrize("missing", MISSING, ids=["fused", "apart"])
@pytest.mark.parametrize("dtype,state,stochastic", KINDS)
def test_a_rate_on_the_device_that_a_number_may_not_be_leaves_the_call_out(dtype, state, stochastic, missing):
    run = Run([700, 300, 5000], dtype, None, state, seed=22, no_grad=missing, stochastic=stochastic)
    run.step(lr=1e-3)
    keep = run.snapshot()
    norm = run.opt.state_get().norm
    for i, lr in enumerate((-1e-19, -5e-324, -1.0, math.nan, math.inf, -math.inf)):
        clip = 0.5 if i % 2 else None
        run.opt.step(run.params, run.grads, run.state, on_device(lr), max_norm=clip)
        rec = run.opt.state_get()
        assert (rec.step, rec.skipped, rec.clip_coef) == (1, i + 1, 0.0), lr
        if clip:  # the call did take one
            norm = math.sqrt(sum(float(g.double().square().sum()) for g in run.grads if g is not None))
        assert rec.norm == pytest.approx(norm, rel=1e-12)
        assert all(torch.equal(x, y) for x, y in zip(run.snapshot(), keep)), lr
    run.draw(1)
    run.step(lr=on_device(1e-3), max_norm=0.5)
    assert run.opt.state_get().step == 2
    run.close()


@pytest.mark.parametrize("missing", MISSING, ids=["fused", "apart"])
def test_a_schedule_under_a_graph_may_end_at_and_below_zero(missing):
    a, b = (Run([700, 300, 5000], "bf16", None, "e4m3", seed=23, no_grad=missing) for _ in range(2))
    lr = on_device(0.0)
    plan = a.opt.prepare(a.params, a.grads, a.state)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=torch.cuda.Stream(DEV)):
        plan.run(lr, max_norm=0.5, seed=3)
    for t, rate in enumerate((1e-2, 1e-3, 0.0, -0.0, -1e-19, 1e-3)):
        for r in (a, b):
            r.draw(t)
        lr.fill_(rate)
        graph.replay()
        torch.cuda.synchronize()
        if rate >= 0.0:
            b.opt.step(b.params, b.grads, b.state, abs(rate), max_norm=0.5, seed=3)
        assert all(torch.equal(x, y) for x, y in zip(a.snapshot(), b.snapshot())), (t, rate)
    rec = a.opt.state_get()
    assert (rec.step, rec.skipped) == (5, 1) and rec.step == b.opt.state_get().step
    a.close()
    b.close()


def test_the_same_numbers_are_refused_on_the_host():
    run = Run([300], "f32", seed=24)
    for lr in (-1e-19, -5e-324, -1.0, math.nan, math.inf, -math.inf):
        with pytest.raises(EditOuterError, match="lr must be finite"):
            run.opt.step(run.params, run.grads, run.state, lr)
    assert run.opt.state_get().step == 0
    run.step(lr=np.float64(-0.0))
    run.close()
