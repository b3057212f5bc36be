"""The AdamW step over many tensors against its formulas in 64 bits (GPU)."""
import numpy as np
import pytest
import torch

import adamw_reference as ref
from paper_2412_07210_amd import AdamW, AdamWConfig, AdamWState, EditOuterError
from paper_2412_07210_amd.outer import EDIT_EINVAL

pytestmark = pytest.mark.gpu

DEV = torch.device("cuda:0")
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
# empty, single, ends inside and at scale blocks and at the kernels' blocks
SIZES = [1, 0, 7, 8, 9, 255, 256, 257, 511, 2047, 2048, 2049, 5003, 0, 33000]


def randn(n, seed, std=1.0):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    return torch.empty(n, device=DEV).normal_(0.0, std, generator=gen)


class Run:
    """Tensors as views at odd offsets of flat buffers, guarded on both sides, and the
    64-bit step beside the handle's, from the same values every time."""

    def __init__(self, sizes, dtype="bf16", grad_dtype=None, state="f32", seed=0, no_grad=(), gap=3, std=1e-2, **more):
        self.cfg = AdamWConfig(list(sizes), dtype, grad_dtype, state, **{**dict(
            betas=(0.9, 0.95), weight_decay=0.1, decay=[0.0 if k % 3 == 1 else 1.0 + k for k in range(len(sizes))]), **more})
        self.opt = AdamW(self.cfg, DEV)
        self.sizes, self.seed, self.std, self.no_grad = list(sizes), seed, std, set(no_grad)
        total = sum(n + gap for n in sizes) + gap
        self.flat_p = randn(total, seed, 0.02).to(TYPES[dtype])
        self.flat_g = torch.zeros(total, dtype=TYPES[grad_dtype or dtype], device=DEV)
        self.at = np.cumsum([gap] + [n + gap for n in sizes])[:-1]
        self.params = [self.flat_p[a:a + n] for a, n in zip(self.at, sizes)]
        self.grads = [None if k in self.no_grad else self.flat_g[a:a + n] for k, (a, n) in enumerate(zip(self.at, sizes))]
        self.state = self.opt.new_state()
        self.held = state == "e4m3"
        self.draw(0)

    def draw(self, t):
        """New gradients: noise, zeros and a few large ones."""
        g = randn(self.flat_g.numel(), 1000 * self.seed + t + 1, self.std)
        g[::7] *= 30.0
        g[3::11] = 0.0
        self.flat_g.copy_(g)

    def numpy_states(self, k):
        s = self.state
        if self.held:
            return [ref.values(c[k], x[k]) for c, x in ((s.exp_avg, s.exp_avg_scale), (s.exp_avg_sq, s.exp_avg_sq_scale))]
        return [x[k].double().cpu().numpy() for x in (s.exp_avg, s.exp_avg_sq)]

    def snapshot(self):
        s = self.state
        every = [*s.exp_avg, *s.exp_avg_sq, *(s.exp_avg_scale or []), *(s.exp_avg_sq_scale or [])]
        return [self.flat_p.clone()] + [x.view(torch.uint8).clone() if x.dtype == torch.float8_e4m3fn else x.clone() for x in every]

    def step(self, lr=3e-3, max_norm=None, seed=0, **more):
        """One step, and the check of everything it wrote."""
        cfg = self.cfg
        before = self.flat_p.clone()
        olds = [self.numpy_states(k) for k in range(len(self.sizes))]
        kept = self.snapshot()
        t = self.opt.state_get().step + 1
        self.opt.step(self.params, self.grads, self.state, lr, max_norm=max_norm, seed=seed, **more)
        rec = self.opt.state_get()
        assert rec.step == t
        clip = 1.0
        if max_norm is not None:
            s = sum(float(g.double().cpu().square().sum()) for g in self.grads if g is not None)
            assert rec.norm == pytest.approx(s ** 0.5, rel=1e-12)
            clip = min(1.0, max_norm / (s ** 0.5 + 1e-6))
            assert abs(rec.clip_coef - clip) <= 2.0 ** -24 * clip * 1.001
            clip = rec.clip_coef
        lr = float(lr)
        for k, n in enumerate(self.sizes):
            if n == 0 or k in self.no_grad:
                continue
            what = f"tensor {k} of {n} at t = {t}"
            old = before[self.at[k]:self.at[k] + n].double().cpu().numpy()
            p, m, v, step, terms = ref.step64(old, self.grads[k].float().cpu().numpy(), *olds[k], t, lr, cfg.betas, cfg.eps,
                                       cfg.weight_decay * np.float32(cfg.decay[k]), clip)
            first, second = ref.words(seed, t, k, np.arange(n))
            s = self.state
            if self.held:
                ref.assert_held(s.exp_avg[k], s.exp_avg_scale[k], m.astype(np.float32), first, False, what + " m")
                ref.assert_held(s.exp_avg_sq[k], s.exp_avg_sq_scale[k], v.astype(np.float32), first, True, what + " v")
            else:
                ref.assert_states(s.exp_avg[k], m, what + " m", terms)
                ref.assert_states(s.exp_avg_sq[k], v, what + " v")
            ref.assert_params(self.params[k], p, step, what + " p", second if cfg.stochastic else None)
        # what is between the tensors, and tensors without a gradient, stay
        mask = torch.ones(len(before), dtype=torch.bool, device=DEV)
        for k, n in enumerate(self.sizes):
            if k not in self.no_grad:
                mask[self.at[k]:self.at[k] + n] = False
        assert torch.equal(self.flat_p[mask], before[mask])
        now = self.snapshot()
        for k in self.no_grad:
            for i in range(1, len(now), len(self.sizes)):
                assert torch.equal(now[i + k], kept[i + k])

    def close(self):
        self.opt.close()


VARIANTS = [(d, g, s, r) for d in ("bf16", "f32") for g in ("bf16", "f32") for s in ("f32", "e4m3")
            for r in ((False, True) if d == "bf16" else (False,))]


@pytest.mark.parametrize("clip", [None, 0.5])
@pytest.mark.parametrize("dtype,grad,state,stochastic", VARIANTS)
def test_steps(dtype, grad, state, stochastic, clip):
    """Four steps from zero states, every variant of the kernel."""
    run = Run(SIZES, dtype, grad, state, seed=3, stochastic=stochastic)
    for t in range(4):
        run.draw(t)
        run.step(max_norm=clip, seed=2 ** 63 + 11 * t)
    run.close()


@pytest.mark.parametrize("sizes,seed", [([40, 300], 1), ([5000] * 3, 2), ([100003], 3)])
@pytest.mark.parametrize("state", ["f32", "e4m3"])
@pytest.mark.parametrize("over", [
    dict(betas=(0.0, 0.0)), dict(betas=(0.9, 0.999), eps=1e-12), dict(weight_decay=0.0), dict(eps=1.0), dict(betas=(0.99, 0.5)),
], ids=str)
def test_hyper_parameters(state, over, sizes, seed):
    run = Run(sizes, "f32", None, state, seed=seed, **over)
    for t, lr in enumerate((1.0, 0.0, 1e-3, 1e-30)):
        run.draw(t)
        run.step(lr=lr)
    run.close()


def test_elements_without_a_gradient_stay_at_any_rate():
    """m = v = 0: a quotient of zero, however large or small the rate is."""
    p, g = [randn(700, 1)], [torch.zeros(700, device=DEV)]
    with AdamW(AdamWConfig([700], "f32", weight_decay=0.0, eps=1e-12), DEV) as o:
        s, keep = o.new_state(), p[0].clone()
        for lr in (0.0, 1e-300, 1e-3, 1e30, 1e300):
            o.step(p, g, s, lr)
            assert torch.equal(p[0], keep), lr


@pytest.mark.parametrize("std", [1e-18, 1e-9, 1e3, 1e15])
@pytest.mark.parametrize("state", ["f32", "e4m3"])
def test_gradients_of_any_size(state, std):
    """Squares near both ends of fp32's range, and scales at their lower end."""
    run = Run([3000, 257], "f32", None, state, seed=4, std=std)
    for t in range(3):
        run.draw(t)
        run.step()
    run.close()


@pytest.mark.parametrize("offset", range(8))
@pytest.mark.parametrize("dtype,state", [("bf16", "e4m3"), ("f32", "f32")])
def test_every_alignment(dtype, state, offset):
    run = Run([700, 2048 + offset], dtype, None, state, seed=offset, gap=offset)
    run.step()
    run.draw(1)
    run.step(max_norm=1.0)
    run.close()


@pytest.mark.parametrize("count", [55, 56, 57, 113, 192, 193, 400])
@pytest.mark.parametrize("state", ["f32", "e4m3"])
def test_many_tensors(state, count):
    """More tensors than one launch of either pass takes; some empty, some without a gradient."""
    rng = np.random.default_rng(count)
    sizes = [int(n) for n in rng.integers(0, 700, count)]
    run = Run(sizes, "bf16", None, state, seed=count, no_grad=[0, 5, 56, count - 1] if count > 56 else [5], stochastic=True)
    for t in range(2):
        run.draw(t)
        run.step(max_norm=0.3, seed=t)
    run.close()


def test_tables_without_a_gradient():
    """Whole launches' tensors without a gradient, and then all of them: t goes on."""
    run = Run([100] * 130, seed=6, no_grad=range(10, 125))
    run.step(max_norm=0.01)
    run.close()
    run = Run([100] * 130, seed=6, no_grad=range(130))
    run.step(max_norm=1.0)
    assert run.opt.state_get().clip_coef == 1.0 and run.opt.state_get().norm == 0.0
    assert float(run.opt.sum_squares(run.grads)) == 0.0
    run.close()


@pytest.mark.parametrize("large", [0, 3_000_000])
@pytest.mark.parametrize("dtype,state", [("bf16", "e4m3"), ("f32", "f32")])
def test_calls_with_and_without_every_gradient(dtype, state, large):
    """Few blocks decide in the update pass where every tensor has a gradient, and in a
    launch before it otherwise (as many blocks do): t counts on from one to the other,
    clipped or not, left out or not, set anew or not."""
    sizes = [700, 0, 5000, 60, 300 + large]
    run = Run(sizes, dtype, None, state, seed=17, stochastic=dtype == "bf16")
    full = list(run.grads)
    for t, missing in enumerate([[], [2], [], [], [0, 3], [4], [], [2]]):
        run.draw(t)
        run.no_grad = set(missing)
        run.grads = [None if k in missing else g for k, g in enumerate(full)]
        run.step(max_norm=0.2 if t % 3 == 1 else None, seed=t)
        if t in (3, 4):  # left out in between
            keep = run.snapshot()
            full[2 if t == 3 else 4][7] = float("inf")
            run.opt.step(run.params, run.grads, run.state, 1e-2, max_norm=1.0)
            assert run.opt.state_get().step == t + 1 and run.opt.state_get().skipped == t - 2
            assert all(torch.equal(x, y) for x, y in zip(run.snapshot(), keep))
        if t == 5:
            run.opt.state_set(6)
    assert run.opt.state_get().step == 8
    run.close()


def test_no_tensors():
    for sizes in ([], [0], [0, 0]):
        run = Run(sizes, seed=1)
        run.step()
        run.step(max_norm=1.0)
        run.close()


# ---- the norm -----------------------------------------------------------------------

@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("sizes", [[1], [5], [2048], [8191, 8192, 8193], SIZES, [3_000_001, 1, 70_000], [999] * 450],
                         ids=["1", "5", "2048", "8191..8193", "SIZES", "ragged", "450"])
def test_sum_squares(dtype, sizes):
    """Against fp64: squares of bf16 and fp32 values are exact there, sums of n of them
    in any order are off by n 2^-53 at most."""
    run = Run(sizes, dtype, seed=7)
    want = sum(float(g.double().square().sum()) for g in run.grads)
    out = torch.full((1,), -1.0, dtype=torch.float64, device=DEV)
    assert run.opt.sum_squares(run.grads, out) is out
    assert abs(float(out) - want) <= 2 * sum(sizes) * 2.0 ** -53 * want
    assert float(run.opt.sum_squares(run.grads)) == float(out)
    assert run.opt.state_get().step == 0
    run.close()


def test_shards_share_a_norm():
    """Two handles with half the tensors each, clipped by the norm of all, step as one handle does."""
    sizes = [4000, 2500, 777, 12]
    whole, a, b = (Run(s, "f32", state="f32", seed=8) for s in (sizes, sizes[:2], sizes[2:]))
    for part, ks in ((a, range(2)), (b, range(2, 4))):
        for i, k in enumerate(ks):
            part.params[i].copy_(whole.params[k])
            part.grads[i].copy_(whole.grads[k])
        part.opt.cfg.decay = part.cfg.decay
    whole.opt.step(whole.params, whole.grads, whole.state, 1e-2, max_norm=0.1)
    s = a.opt.sum_squares(a.grads) + b.opt.sum_squares(b.grads)
    for part in (a, b):
        part.opt.step(part.params, part.grads, part.state, 1e-2, max_norm=0.1, sumsq=s)
        assert part.opt.state_get().clip_coef == whole.opt.state_get().clip_coef < 1.0
        assert part.opt.state_get().norm == pytest.approx(whole.opt.state_get().norm, rel=1e-12)
    for k, x in enumerate([*a.state.exp_avg, *b.state.exp_avg]):
        assert torch.equal(x, whole.state.exp_avg[k])
    for r in (whole, a, b):
        r.close()


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("state", ["f32", "e4m3"])
def test_a_gradient_that_is_not_finite_leaves_a_clipped_call_out(state, bad):
    run = Run([300, 5000], "bf16", None, state, seed=9)
    run.step(max_norm=1.0)
    keep = run.snapshot()
    run.grads[1][4321] = bad
    run.opt.step(run.params, run.grads, run.state, 1e-2, max_norm=1.0)
    run.opt.step(run.params, run.grads, run.state, 1e-2, sumsq=torch.full((1,), bad, dtype=torch.float64, device=DEV))
    rec = run.opt.state_get()
    assert (rec.step, rec.skipped, rec.clip_coef) == (1, 2, 0.0) and not np.isfinite(rec.norm)
    assert all(torch.equal(x, y) for x, y in zip(run.snapshot(), keep))
    run.draw(5)
    run.step(max_norm=1.0)
    assert run.opt.state_get().step == 2
    run.close()


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
@pytest.mark.parametrize("dtype,state,stochastic", [("bf16", "e4m3", True), ("f32", "e4m3", False), ("bf16", "f32", True)])
def test_without_a_clip_it_stays_in_its_element(dtype, state, stochastic, bad):
    """The element's p, m and v are NaN (or infinite, in fp32); all others are as they would be."""
    run, other = (Run([5000, 300], dtype, "f32", state, seed=10, stochastic=stochastic) for _ in range(2))
    spots = [0, 255, 256, 4999]
    for r in (run, other):
        r.grads[0][spots] = 0.0  # so that they are not their block's largest
        r.step()
        r.draw(1)
    run.grads[0][spots] = bad
    other.grads[0][spots] = 0.0
    for r in (run, other):
        r.opt.step(r.params, r.grads, r.state, 1e-2)
    torch.cuda.synchronize()
    fine = torch.ones(5000, dtype=torch.bool, device=DEV)
    fine[spots] = False
    assert torch.isnan(run.params[0][spots].float()).all()
    for x in (run.state.exp_avg[0], run.state.exp_avg_sq[0]):
        assert not torch.isfinite(x[spots].float()).any()
    assert torch.equal(run.params[0][fine], other.params[0][fine]) and torch.equal(run.params[1], other.params[1])
    for x, y in ((run.state.exp_avg, other.state.exp_avg), (run.state.exp_avg_sq, other.state.exp_avg_sq)):
        assert torch.equal(x[0].float()[fine], y[0].float()[fine])
    if state == "e4m3":
        assert torch.equal(run.state.exp_avg_scale[0], other.state.exp_avg_scale[0])
        assert torch.equal(run.state.exp_avg_sq_scale[0], other.state.exp_avg_sq_scale[0])
    run.close()
    other.close()


# ---- 8-bit states -------------------------------------------------------------------

@pytest.mark.parametrize("std", [1e-30, 1e-12, 1.0, 1e20])
def test_pack_and_unpack(std):
    sizes = [1, 255, 0, 256, 257, 5000, 70_001]
    opt = AdamW(AdamWConfig(sizes, state="e4m3"), DEV)
    m = [randn(n, 20 + k, std) for k, n in enumerate(sizes)]
    v = [randn(n, 40 + k, 1.0).mul_(4.0).exp_().mul_(std) for k, n in enumerate(sizes)]
    m[5][100:600] = 0.0  # a whole block among them
    m[4][3], v[4][256] = float("nan"), float("inf")
    m = [torch.cat([x, x.new_zeros(4)])[:len(x)] for x in m]  # aligned copies
    state = opt.pack(m, v, seed=77)
    back = opt.unpack(state)
    torch.cuda.synchronize()
    for k, n in enumerate(sizes):
        if n == 0:
            continue
        w, _ = ref.words(77, 0, k, np.arange(n))
        for x, codes, scale, y, second in ((m[k], state.exp_avg[k], state.exp_avg_scale[k], back[0][k], False),
                                           (v[k], state.exp_avg_sq[k], state.exp_avg_sq_scale[k], back[1][k], True)):
            x = x.cpu().numpy()
            value, s = ref.held(x, w, second)
            assert (scale.cpu().double().numpy() == s).all(), f"{k}"
            got = codes.float().cpu().double().numpy()
            assert np.array_equal(got, value, equal_nan=True), f"{k}: {(got != value).sum()}"
            want = (value * np.repeat(s, 256)[:n]).astype(np.float32)
            assert np.array_equal(y.cpu().numpy(), want, equal_nan=True)
    other = opt.pack(m, v, seed=78)
    assert (other.exp_avg[6].view(torch.uint8) != state.exp_avg[6].view(torch.uint8)).any()
    opt.close()


def test_held_v_follows_its_mean():
    """v in 8 bits under a constant g^2 far from where v began: right on average.  With
    g the same every step and beta2 = 0.99, v_t = g^2 + (v_0 - g^2) 0.99^t; rounding adds
    noise without a mean, of a relative variance of at most (1 - beta2) 2^-3 a step, so
    the mean over n elements is off by less than 6 sqrt(0.125 / n) of v (a step's
    noise decays with v: the sum of its variances is at most 2^-3 / 2)."""
    n = 65536
    opt = AdamW(AdamWConfig([n], "f32", state="e4m3", betas=(0.9, 0.99)), DEV)
    p, g = [torch.zeros(n, device=DEV)], [torch.full((n,), 1e-3, device=DEV)]
    for v0 in (1.6e-5, 1e-9):
        state = opt.pack([torch.zeros(n, device=DEV)], [torch.full((n,), v0, device=DEV)], seed=1)
        plan = opt.prepare(p, g, state)
        for t in range(150):
            plan.run(0.0, seed=5)
        got = float(opt.unpack(state)[1][0].double().mean())
        want = 1e-6 + (v0 - 1e-6) * 0.99 ** 150
        assert abs(got - want) <= 6 * np.sqrt(0.125 / n) * max(want, v0 * 0.99 ** 150), (v0, got, want)
    opt.close()


def test_stochastic_parameters_move_on_average():
    """A bf16 p whose steps are a 64th of its spacing: nearest keeps it, stochastic moves it on average."""
    n, steps = 65536, 32
    lr = 2.0 ** -7 / 64  # p = 1: spacing 2^-7 above
    got = {}
    for stochastic in (False, True):
        opt = AdamW(AdamWConfig([n], "bf16", state="f32", weight_decay=0.0, stochastic=stochastic), DEV)
        p = [torch.ones(n, dtype=torch.bfloat16, device=DEV)]
        g = [torch.full((n,), -1.0, dtype=torch.bfloat16, device=DEV)]  # update of one, whatever t
        plan = opt.prepare(p, g, opt.new_state())
        for t in range(steps):
            plan.run(lr, seed=3)
        got[stochastic] = float(p[0].double().mean())
        opt.close()
    assert got[False] == 1.0
    # each step rounds up with probability 1 / 64: mean steps * lr, variance below steps / 64 spacings^2 an element
    assert abs(got[True] - 1.0 - steps * lr) <= 6 * 2.0 ** -7 * np.sqrt(steps / 64 / n)


# ---- calls ---------------------------------------------------------------------------

@pytest.mark.parametrize("state", ["f32", "e4m3"])
def test_graph_replays_go_on(state):
    """A captured step, clipped, with the rate on the device, replayed with other
    gradients and rates and eager steps in between: as eager steps, bit for bit."""
    a, b = (Run([3000, 100, 70_000], "bf16", None, state, seed=11, stochastic=True) for _ in range(2))
    lr = torch.zeros(1, dtype=torch.float64, device=DEV)
    plan = a.opt.prepare(a.params, a.grads, a.state)
    plan.run(1e-2, max_norm=1.0, seed=9)
    b.opt.step(b.params, b.grads, b.state, 1e-2, max_norm=1.0, seed=9)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=torch.cuda.Stream(DEV)):
        plan.run(lr, max_norm=1.0, seed=9)
    assert all(torch.equal(x, y) for x, y in zip(a.snapshot(), b.snapshot()))
    for t in range(4):
        for r in (a, b):
            r.draw(t + 1)
        if t == 2:
            a.grads[0][5] = b.grads[0][5] = float("nan")  # left out, on both sides
        lr.fill_(1e-2 / (t + 1))
        graph.replay()
        torch.cuda.synchronize()
        b.opt.step(b.params, b.grads, b.state, 1e-2 / (t + 1), max_norm=1.0, seed=9)
        assert a.opt.state_get() == b.opt.state_get() or t == 2
        assert all(torch.equal(x, y) for x, y in zip(a.snapshot(), b.snapshot())), f"replay {t}"
        if t == 1:
            for r in (a, b):
                r.step(lr=1e-3, seed=1)
    assert a.opt.state_get().step == 5 and a.opt.state_get().skipped == 1
    a.close()
    b.close()


def test_two_graphs_of_one_handle():
    """The norm's workspace and the record belong to the handle: graphs replayed one after the other."""
    a, b = (Run([30_000, 77], "f32", None, "e4m3", seed=12) for _ in range(2))
    plans = [a.opt.prepare(a.params, a.grads, a.state) for _ in range(2)]
    graphs = []
    torch.cuda.synchronize()
    for plan, norm in zip(plans, (0.5, 5.0)):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1], stream=torch.cuda.Stream(DEV)):
            plan.run(1e-2, max_norm=norm)
    for t in range(4):
        for r in (a, b):
            r.draw(t)
        graphs[t % 2].replay()
        b.opt.step(b.params, b.grads, b.state, 1e-2, max_norm=(0.5, 5.0)[t % 2])
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(a.snapshot(), b.snapshot())), f"replay {t}"
    a.close()
    b.close()


def test_another_stream_and_runs_agree():
    a, b = (Run(SIZES, "bf16", None, "e4m3", seed=13, stochastic=True) for _ in range(2))
    side = torch.cuda.Stream(DEV)
    for t in range(3):
        for r in (a, b):
            r.draw(t)
        side.wait_stream(torch.cuda.current_stream(DEV))
        a.opt.step(a.params, a.grads, a.state, 1e-2, max_norm=1.0, seed=t, stream=side)
        torch.cuda.current_stream(DEV).wait_stream(side)
        b.opt.step(b.params, b.grads, b.state, 1e-2, max_norm=1.0, seed=t)
    assert all(torch.equal(x, y) for x, y in zip(a.snapshot(), b.snapshot()))
    a.close()
    b.close()


def test_resumed_run_goes_on_bit_for_bit():
    a, b = (Run([5000, 3], "bf16", None, "e4m3", seed=14, stochastic=True) for _ in range(2))
    for r in (a, b):
        for t in range(2):
            r.opt.step(r.params, r.grads, r.state, 1e-2, seed=4)
    b.opt.close()
    b.opt = AdamW(b.cfg, DEV)
    b.opt.state_set(2)
    for r in (a, b):
        r.opt.step(r.params, r.grads, r.state, 1e-2, seed=4)
    assert all(torch.equal(x, y) for x, y in zip(a.snapshot(), b.snapshot()))
    a.opt.step(a.params, a.grads, a.state, 1e-2, seed=4)
    b.opt.step(b.params, b.grads, b.state, 1e-2, seed=5)
    assert not all(torch.equal(x, y) for x, y in zip(a.snapshot(), b.snapshot()))
    a.close()
    b.close()


def test_refusals_change_nothing():
    run = Run([600, 700], "bf16", None, "e4m3", seed=15)
    p, g, s = run.params, run.grads, run.state
    keep = run.snapshot()
    flat8 = torch.zeros(4096, dtype=torch.uint8, device=DEV).view(torch.float8_e4m3fn)
    cases = [
        (([p[0], run.flat_p[at:at + 700]], g, s), "overlap") for at in (int(run.at[0]), int(run.at[0]) + 599)
    ] + [
        ((p, [run.flat_p[int(run.at[0]):int(run.at[0]) + 600], g[1]], s), "must not overlap what is written"),
        ((p, g, AdamWState([flat8[1:601], s.exp_avg[1]], s.exp_avg_sq, s.exp_avg_scale, s.exp_avg_sq_scale)), "16-byte aligned"),
        ((p, g, AdamWState(s.exp_avg, s.exp_avg, s.exp_avg_scale, s.exp_avg_sq_scale)), "overlap"),
        ((p, g, AdamWState(s.exp_avg, s.exp_avg_sq, s.exp_avg_scale, s.exp_avg_scale)), "overlap"),
    ]
    for args, needle in cases:
        with pytest.raises(EditOuterError, match=needle) as e:
            run.opt.step(*args, 1e-3)
        assert e.value.status == EDIT_EINVAL
    for lr in (-1e-3, float("nan"), float("inf")):
        with pytest.raises(EditOuterError, match="lr"):
            run.opt.step(p, g, s, lr)
    with pytest.raises(EditOuterError, match="step must be"):
        run.opt.state_set(-1)
    with pytest.raises(EditOuterError, match="step must be"):
        run.opt.state_set(2 ** 62 + 1)
    with pytest.raises(ValueError, match=r"params\[0\]"):
        run.opt.step([p[0].cpu(), p[1]], g, s, 1e-3)
    assert run.opt.state_get().step == 0
    assert all(torch.equal(x, y) for x, y in zip(run.snapshot(), keep))
    # the same gradient for two tensors is read twice, and that is all
    same = run.flat_g[int(run.at[1]):int(run.at[1]) + 600]
    run.grads[0] = same
    run.step()
    run.close()
    plain = AdamW(AdamWConfig([600], "f32"), DEV)
    with pytest.raises(EditOuterError, match="fp32"):
        plain.pack([torch.zeros(600, device=DEV)], [torch.zeros(600, device=DEV)], plain.new_state())
    plain.close()
    with pytest.raises(EditOuterError, match="NULL handle"):
        plain.step([torch.zeros(600, device=DEV)], [torch.zeros(600, device=DEV)], plain.new_state(), 1e-3)


@pytest.mark.parametrize("over", ["param", "exp_avg", "exp_avg_sq"])
def test_numbers_read_on_the_device_are_not_written(over):
    run = Run([600, 700], "f32", None, "f32", seed=16)
    keep = run.snapshot()
    buffer = {"param": run.flat_p[int(run.at[0]):], "exp_avg": run.state.exp_avg[1], "exp_avg_sq": run.state.exp_avg_sq[0]}[over]
    skip = buffer.data_ptr() % 8 // 4
    number = buffer[skip + 200:skip + 202].view(torch.float64)
    for lr, sumsq in ((number, None), (1e-3, number)):
        with pytest.raises(EditOuterError, match="lr_device and sumsq must not overlap") as e:
            run.opt.step(run.params, run.grads, run.state, lr, sumsq=sumsq)
        assert e.value.status == EDIT_EINVAL
    assert run.opt.state_get().step == 0
    assert all(torch.equal(x, y) for x, y in zip(run.snapshot(), keep))
    # between the buffers, as an allocator may place it, is another matter
    apart = torch.tensor([1e-3], dtype=torch.float64, device=DEV)
    run.opt.step(run.params, run.grads, run.state, apart)
    assert run.opt.state_get().step == 1
    run.close()


@pytest.mark.skipif(torch.cuda.device_count() < 2, reason="needs two devices")
def test_beside_another_current_device():
    run, other = (Run([5000], seed=16) for _ in range(2))
    run.opt.step(run.params, run.grads, run.state, 1e-2, max_norm=1.0)
    with torch.cuda.device(1):
        other.opt.step(other.params, other.grads, other.state, 1e-2, max_norm=1.0)
        assert torch.cuda.current_device() == 1
    torch.cuda.synchronize(DEV)
    assert torch.equal(run.flat_p, other.flat_p)
    run.close()
    other.close()
