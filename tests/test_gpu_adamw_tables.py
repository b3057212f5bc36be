"""Calls of few blocks over more tensors than one launch takes, every one with a
gradient: the decision in the update passes of several launches (GPU)."""
import numpy as np
import pytest
import torch

from test_gpu_adamw import DEV, Run

pytestmark = pytest.mark.gpu

# (dtype, state, elements of a block of the update pass)
KINDS = [("f32", "f32", 256), ("bf16", "f32", 256), ("f32", "e4m3", 512), ("bf16", "e4m3", 1024)]


def sizes_of(count, block, seed):
    """Tensors of up to three blocks, empty ones among them, 2048 blocks at most in all."""
    rng = np.random.default_rng(seed)
    sizes = [int(n) for n in rng.integers(0, 3 * block if count < 400 else 2 * block, count)]
    sizes[3] = sizes[count // 2] = 0
    sizes[count - 1] = max(1, sizes[count - 1])
    assert 1 < sum(-(-n // block) for n in sizes) <= 2048
    return sizes


@pytest.mark.parametrize("count", [56, 57, 112, 113, 400])
@pytest.mark.parametrize("dtype,state,block", KINDS)
def test_steps_of_several_launches(dtype, state, block, count):
    """Clipped and not, left out in between, set anew, with a gradient missing (which
    takes the decision before the update pass) and whole again: every tensor's t is
    the call's, as its bias corrections and random numbers show."""
    run = Run(sizes_of(count, block, count), dtype, None, state, seed=count, stochastic=dtype == "bf16")
    full = list(run.grads)
    for t in range(6):
        run.draw(t)
        missing = {3: {count - 2}, 4: {0, 1}}.get(t, set())
        run.no_grad, run.grads = missing, [None if k in missing else g for k, g in enumerate(full)]
        run.step(max_norm=0.2 if t % 2 else None, seed=t)
        if t == 1:  # a gradient of the first launch's tensors, and one of the last's
            for k in (0, count - 1):
                n = next(i for i in range(k, count) if run.sizes[i]) if k == 0 else k
                keep = run.snapshot()
                full[n][0] = float("nan")
                run.opt.step(run.params, run.grads, run.state, 1e-2, max_norm=1.0)
                full[n][0] = 0.0
                assert all(torch.equal(x, y) for x, y in zip(run.snapshot(), keep))
            assert run.opt.state_get().step == 2 and run.opt.state_get().skipped == 2
        if t == 2:
            run.opt.state_set(2 ** 33)
    assert run.opt.state_get().step == 2 ** 33 + 3
    run.close()


@pytest.mark.parametrize("count", [57, 400])
@pytest.mark.parametrize("dtype,state,block", [KINDS[0], KINDS[3]])
def test_replays_of_several_launches(dtype, state, block, count):
    sizes = sizes_of(count, block, count)
    a, b = (Run(sizes, dtype, None, state, seed=25, stochastic=dtype == "bf16") for _ in range(2))
    plan = a.opt.prepare(a.params, a.grads, a.state)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=torch.cuda.Stream(DEV)):
        plan.run(1e-2, max_norm=0.5, seed=7)
        plan.run(1e-3, seed=8)
    for t in range(4):
        for r in (a, b):
            r.draw(t)
        if t == 2:
            for r in (a, b):
                r.opt.step(r.params, r.grads, r.state, 1e-3, seed=1)
        graph.replay()
        torch.cuda.synchronize()
        b.opt.step(b.params, b.grads, b.state, 1e-2, max_norm=0.5, seed=7)
        b.opt.step(b.params, b.grads, b.state, 1e-3, seed=8)
        assert all(torch.equal(x, y) for x, y in zip(a.snapshot(), b.snapshot())), f"replay {t}"
        assert a.opt.state_get() == b.opt.state_get()
    assert a.opt.state_get().step == 9
    a.close()
    b.close()
