"""Orthogonalised updates against the plain 64-bit implementation (GPU):
O(U) by itself, the local step and the outer step, over shapes, spectra,
offsets, types, precisions and the calls that the header allows.  Tolerances
are derived in ortho_reference.py.
"""
import math

import pytest
import torch

from ortho_reference import (DEFAULT, assert_o_close, half_step, layout, mask_of, matrix, o_tolerance, ortho64)
from paper_2412_07210_amd import AE, GC, ONE_PASS, WA, EditOuter, EditOuterError, OrthoConfig, Orthogonalizer, OuterConfig

pytestmark = pytest.mark.gpu

DEV = torch.device("cuda:0")
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
KINDS = [("bf16", "fast"), ("f32", "full"), ("f32", "fast"), ("bf16", "full")]


def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def _randn(n, seed, std=1.0):
    return torch.empty(n, device=DEV).normal_(0.0, std, generator=_gen(seed))


def _ortho(numel, matrices, dtype, precision=None, **more):
    return Orthogonalizer(OrthoConfig(numel, matrices, dtype=dtype, precision=precision, **more), DEV)


SHAPES = [
    [(1, 1)], [(1, 7), (5, 1), (3, 3)], [(16, 16)], [(64, 64), (65, 63), (63, 65)], [(127, 129), (129, 127)],
    [(128, 128)], [(256, 31), (31, 256)], [(100, 300), (300, 100), (129, 257)], [(513, 1000)], [(1000, 513)],
    [(8, 3000), (3000, 8)], [(96, 7129), (5001, 70)], [(128, 128), (1, 256), (96, 250), (256, 64), (17, 33)], [(250, 96)] * 3,
    [(60, 60), (2, 2)], [(30, 9), (32, 32)], [(640, 640)] * 3, [(1, 4097), (4097, 1)], [(384, 700), (700, 384)] * 2, [(1300, 1290)],
]


@pytest.mark.parametrize("dtype,precision", KINDS)
@pytest.mark.parametrize("shapes", SHAPES, ids=lambda s: "+".join("%dx%d" % x for x in s))
def test_orthogonalize_shapes(shapes, dtype, precision):
    numel, mats = layout(shapes)
    x = _randn(numel, 1).to(TYPES[dtype])
    with _ortho(numel, mats, dtype, precision) as o:
        y = o.orthogonalize(x)
        again = o.orthogonalize(x)
    assert torch.equal(y, again)
    for m in mats:
        assert_o_close(matrix(y, m), ortho64(matrix(x, m)), precision, f"{dtype} {precision} {m}")


@pytest.mark.parametrize("shapes,gaps", [([(500, 29201)], [3]), ([(29192, 504)], [0]), ([(1000, 7592), (7603, 1010)], [0, 8])],
                         ids=["wide", "tall", "both"])
def test_matrices_of_many_tiles(shapes, gaps):
    """Work for every CU at the products' largest tiles, whose edges no side is a multiple of."""
    numel, mats = layout(shapes, gaps)
    x = _randn(numel, 6).to(torch.bfloat16)
    p, m = _randn(numel, 7, 0.02).to(torch.bfloat16), torch.zeros(numel, device=DEV)
    with _ortho(numel, mats, "bf16") as o:
        scales = o.cfg.scales()
        y = o.orthogonalize(x)
        assert torch.equal(y, o.orthogonalize(x))
        ref_p, ref_m, outs = _local_step64(p, x, m, mats, scales, 0.02, 0.9, 0.1, True)
        o.local_step(p, x, m, lr=0.02, mu=0.9, weight_decay=0.1)
    for spec in mats:
        assert_o_close(matrix(y, spec), ortho64(matrix(x, spec)), "fast", f"{spec}")
    _check_step(p, ref_p, mats, outs, [0.02 * abs(s) for s in scales], "fast", "local")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("shape", [(4001, 4100), (2900, 2850)])
def test_last_tiles_in_pieces(shape, dtype):
    """A few tiles more than run at a time (528 of 128, 1035 of 64): the last ones' sums are taken in pieces."""
    numel, mats = layout([shape, (90, 70)], [5, 0])
    x = _randn(numel, 8).to(TYPES[dtype])
    with _ortho(numel, mats, dtype) as o:
        y = o.orthogonalize(x)
        assert torch.equal(y, o.orthogonalize(x))
    for spec in mats:
        assert_o_close(matrix(y, spec), ortho64(matrix(x, spec)), "full" if dtype == "f32" else "fast", f"{dtype} {spec}")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_odd_offsets_and_elements_of_no_matrix(dtype):
    """Matrices at odd offsets behind gaps of 1 to 5 elements; what lies between them stays as it was."""
    numel, mats = layout([(33, 47), (64, 64), (5, 130), (130, 70)], gaps=[1, 3, 5, 2], tail=7)
    x = _randn(numel, 2).to(TYPES[dtype])
    outside = ~mask_of(numel, mats, DEV)
    x[outside] = math.nan  # neither read ...
    with _ortho(numel, mats, dtype) as o:
        kept = torch.full_like(x, 7.0)
        o.orthogonalize(x, kept)
        fresh = o.orthogonalize(x)
        where = x.clone()
        assert o.orthogonalize(where, where) is where  # in place
    assert bool((kept[outside] == 7.0).all())  # ... nor written
    assert bool((fresh[outside] == 0.0).all())
    assert bool(where[outside].isnan().all())
    inside = ~outside
    assert torch.equal(kept[inside], fresh[inside]) and torch.equal(kept[inside], where[inside])
    for m in mats:
        assert_o_close(matrix(kept, m), ortho64(matrix(x, m)), "full" if dtype == "f32" else "fast", f"{dtype} {m}")


def _spectrum(kind, rows, cols, seed):
    g = _gen(seed)
    noise = torch.empty(rows, cols, device=DEV).normal_(0.0, 1.0, generator=g)
    if kind == "rank16":
        left = torch.empty(rows, 16, device=DEV).normal_(0.0, 1.0, generator=g)
        right = torch.empty(16, cols, device=DEV).normal_(0.0, 1.0, generator=g)
        return left @ right + 0.1 * noise
    if kind == "rank1":
        return torch.outer(noise[:, 0], noise[0])
    if kind == "one":
        out = torch.zeros_like(noise)
        out[rows // 2, cols // 3] = -3.0
        return out
    if kind == "rows":  # rows of very different size
        return noise * torch.logspace(0, -4, rows, device=DEV)[:, None]
    if kind == "orthogonal":
        return torch.linalg.qr(noise.cpu().double())[0].float().contiguous().to(DEV)
    scale = {"tiny": 1e-30, "huge": 1e30}.get(kind, 1.0)
    return noise * scale


@pytest.mark.parametrize("precision", ["fast", "full"])
@pytest.mark.parametrize("kind", ["rank16", "rank1", "one", "rows", "orthogonal", "tiny", "huge"])
def test_spectra_and_magnitudes(kind, precision):
    rows, cols = 200, 170
    x = _spectrum(kind, rows, cols, 5)
    with _ortho(rows * cols, [(0, rows, cols)], "f32", precision) as o:
        y = o.orthogonalize(x.view(-1))
    assert_o_close(y.view(rows, cols), ortho64(x), precision, f"{kind} {precision}")


def test_subnormal_input():
    """fp32 subnormals have a direction, too."""
    x = (_randn(60 * 50, 8) * 1e-40).view(60, 50)
    assert float(x.abs().max()) > 0
    with _ortho(3000, [(0, 60, 50)], "f32") as o:
        y = o.orthogonalize(x.view(-1))
    assert_o_close(y.view(60, 50), ortho64(x), "full", "subnormal")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
def test_non_finite_matrix_spoils_itself_only(dtype, bad):
    """A NaN or infinity makes its own matrix NaN; the others, a zero matrix among
    them, and the next call with finite values are untouched."""
    numel, mats = layout([(70, 90), (64, 50), (90, 70)])
    x = _randn(numel, 3).to(TYPES[dtype])
    x[mats[1][0]:mats[2][0]] = 0
    with _ortho(numel, mats, dtype) as o:
        clean = o.orthogonalize(x)
        spoilt = x.clone()
        spoilt[mats[0][0] + 11] = bad
        y = o.orthogonalize(spoilt)
        after = o.orthogonalize(x)
    assert bool(matrix(y, mats[0]).isnan().all())
    assert bool((matrix(y, mats[1]) == 0).all())
    assert torch.equal(matrix(y, mats[2]), matrix(clean, mats[2]))
    assert torch.equal(after, clean)


@pytest.mark.parametrize("steps,coef", [
    (1, None), (3, None), (8, None), (4, (1.5, -0.5, 0.0)),
    (3, [(8.29, -23.6, 17.3), (4.1, -2.95, 0.545), (3.9, -2.9, 0.55)]),
])
def test_steps_and_coefficients(steps, coef):
    rows, cols = 150, 260
    x = _randn(rows * cols, 4)
    each = None if coef is None else [coef] * steps if not isinstance(coef, list) else coef
    with _ortho(rows * cols, [(0, rows, cols)], "f32", steps=steps, coefficients=coef) as o:
        y = o.orthogonalize(x)
    ref = ortho64(x.view(rows, cols), steps, each)
    # the polynomials of the last set reach 8.3, three times the default's: three steps count as nine
    assert_o_close(y.view(rows, cols), ref, "full", f"{steps} {coef}", steps=max(steps, 9 if isinstance(coef, list) else 0))


# -------------------------------------------------------------- local step


def _local_step64(p, g, m, mats, scales, lr, mu, decay, nesterov):
    """One step in fp64 from what the tensors hold; (param, momentum) in fp64, and each matrix's O."""
    p, m = p.double(), m.double()
    outs = []
    for spec, s in zip(mats, scales):
        at, r, c = spec
        gm = g[at:at + r * c].double()
        m[at:at + r * c] = mu * m[at:at + r * c] + gm
        mm = m[at:at + r * c]
        o = ortho64((gm + mu * mm if nesterov else mm).view(r, c))
        p[at:at + r * c] = (1 - lr * decay) * p[at:at + r * c] - lr * s * o.reshape(-1)
        outs.append(o)
    return p, m, outs


def _check_step(got, ref, mats, outs, factor, precision, what):
    """Parameters after a step of `factor` * O: O's tolerance times the factor, and one rounding."""
    for spec, o, f in zip(mats, outs, factor):
        y, e = matrix(got, spec), matrix(ref, spec)
        size = float(o.norm())
        tol = o_tolerance(spec[1], spec[2], precision, size) if size else 0.0
        rms = size / math.sqrt(o.numel())
        off = (y.double() - e).abs()
        allowed = 10 * tol * f * o.abs().clamp(min=rms) + half_step(got.dtype) * e.abs() + 1e-30
        assert bool((off <= allowed * (1 + 1e-6)).all()), f"{what} {spec}: {float((off - allowed).max()):.3g} beyond"


@pytest.mark.parametrize("dtype,precision", KINDS)
@pytest.mark.parametrize("nesterov,decay,scale", [(True, 0.1, "rms"), (False, 0.0, "spectral"), (True, 0.0, [1.0, 0.0, -2.0])])
def test_local_steps(dtype, precision, nesterov, decay, scale):
    numel, mats = layout([(96, 200), (300, 64), (77, 77)], gaps=[0, 3, 0], tail=10)
    lr, mu = 0.02, 0.9
    p = _randn(numel, 10, 0.02).to(TYPES[dtype])
    m = torch.zeros(numel, device=DEV)
    outside = ~mask_of(numel, mats, DEV)
    p0 = p.clone()
    m[outside] = 5.0
    with _ortho(numel, mats, dtype, precision, scale=scale) as o:
        scales = o.cfg.scales()
        for step in range(3):
            g = _randn(numel, 20 + step, 1e-3).to(TYPES[dtype])
            g[outside] = math.nan
            ref_p, ref_m, outs = _local_step64(p, g, m, mats, scales, lr, mu, decay, nesterov)
            o.local_step(p, g, m, lr=lr, mu=mu, weight_decay=decay, nesterov=nesterov)
            assert bool(((m.double() - ref_m).abs() <= half_step(torch.float32) * ref_m.abs() * (1 + 1e-6)).all())
            _check_step(p, ref_p, mats, outs, [lr * abs(s) for s in scales], precision, f"step {step}")
    assert torch.equal(p[outside], p0[outside])
    assert bool((m[outside] == 5.0).all())


def test_local_step_with_nothing_to_do():
    """No matrices, empty ones, and lr = 0: parameters stay, the momentum moves."""
    p = _randn(64, 1).to(torch.bfloat16)
    g, m = torch.ones_like(p), torch.zeros(64, device=DEV)
    for mats in ([], [(0, 0, 8), (64, 3, 0)]):
        with _ortho(64, mats, "bf16") as o:
            before = p.clone()
            o.local_step(p, g, m, lr=1.0)
            assert torch.equal(p, before) and bool((m == 0).all())
            assert bool((o.orthogonalize(p) == 0).all())
    with _ortho(0, [], "bf16") as o:
        empty = torch.empty(0, dtype=torch.bfloat16, device=DEV)
        assert o.orthogonalize(empty).numel() == 0
    with _ortho(64, [(0, 8, 8)], "bf16") as o:
        before = p.clone()
        o.local_step(p, g, m, lr=0.0, weight_decay=3.0)
        assert torch.equal(p, before) and bool((m == 1).all())


# -------------------------------------------------------------- outer step


def _outer_pair(K, dtype, numel, **over):
    cfg = OuterConfig(K, [numel], dtype, ema_warmup_rounds=10, **over)
    return cfg, EditOuter(cfg, DEV), EditOuter(cfg, DEV)


def _outer_inputs(K, dtype, numel, seed, stds=None):
    theta = _randn(numel, seed, 0.02)
    b = _randn(numel, seed + 1, 1e-3)
    stds = stds or [1e-3 * (1 + 0.1 * j) for j in range(K)]
    reps = [(theta + _randn(numel, seed + 2 + j, s)).to(TYPES[dtype]) for j, s in enumerate(stds)]
    return theta, b, reps


def _compare_outer(cfg, plain, ortho_handle, o, theta, b, reps, mats, precision, what):
    """A step with orthogonalised matrices against the plain outer step on the same
    inputs: the same decision, EMA and momentum, bit for bit, and the same theta
    and replicas outside the matrices; inside, theta from the plain step's
    momentum in 64 bits."""
    numel = theta.numel()
    t1, b1, r1 = theta.clone(), b.clone(), [r.clone() for r in reps]
    plain.step_layer(0, t1, b1, r1)
    t2, b2, r2 = theta.clone(), b.clone(), [r.clone() for r in reps]
    ortho_handle.step_layer_ortho(0, o, t2, b2, r2)
    sa, sb = plain.state_get(0), ortho_handle.state_get(0)
    for f in ("round", "rolled_back", "z_tested", "synced_norm", "clip_coef"):
        assert getattr(sa, f) == getattr(sb, f) or (sa.synced_norm != sa.synced_norm), (what, f)
    for f in ("ema_mean", "ema_std", "weight", "anomalous"):
        assert getattr(sa, f).tolist() == getattr(sb, f).tolist(), (what, f)
    assert torch.equal(b1, b2), what
    outside = ~mask_of(numel, mats, DEV)
    assert torch.equal(t1[outside], t2[outside]), what
    for x, y in zip(r1, r2):
        assert torch.equal(x[outside], y[outside]), what
        assert torch.equal(y, t2.to(y.dtype)), what
    if sb.rolled_back:
        assert torch.equal(t2, theta) and torch.equal(b2, b), what
        return sb
    # u = rho b' - D, with D from the decision in 64 bits
    d = torch.zeros(numel, dtype=torch.float64, device=DEV)
    for w, r in zip(sb.weight, reps):
        if w != 0:
            d += sb.clip_coef * w * (r.double() - theta.double())
    u = cfg.momentum * (cfg.momentum * b.double() - d) - d
    ref = theta.double()
    outs, factors = [], []
    for spec, s in zip(mats, o.cfg.scales()):
        at, rr, cc = spec
        out = ortho64(u[at:at + rr * cc].view(rr, cc))
        ref[at:at + rr * cc] -= cfg.outer_lr * s * out.reshape(-1)
        outs.append(out)
        factors.append(cfg.outer_lr * abs(s))
    _check_step(t2, ref, mats, outs, factors, precision, what)
    return sb


OUTER_MATS = [[(96, 200), (300, 64), (77, 77)], [(128, 256)]]


@pytest.mark.parametrize("K,dtype", [(1, "bf16"), (2, "f32"), (5, "bf16"), (8, "bf16"), (8, "f32"), (17, "bf16"), (32, "f32")])
@pytest.mark.parametrize("precision", ["full", "fast"])
def test_outer_step(K, dtype, precision):
    for shapes, gaps, tail in ((OUTER_MATS[0], [0, 3, 1], 130), (OUTER_MATS[1], [0], 0)):
        numel, mats = layout(shapes, gaps, tail)
        cfg, plain, handle = _outer_pair(K, dtype, numel, outer_lr=2e-3)
        with plain, handle, _ortho(numel, mats, "f32", precision, scale="rms") as o:
            for rnd in range(2):
                theta, b, reps = _outer_inputs(K, dtype, numel, 100 + 50 * rnd)
                _compare_outer(cfg, plain, handle, o, theta, b, reps, mats, precision, f"K={K} {dtype} round {rnd}")


def _settled(handles, K, numel, std=1e-3):
    g = std * math.sqrt(numel)
    for h in handles:
        h.state_set(0, [g] * K, [0.1 * g] * K, 10)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_outer_step_masks_rollback_and_clip(dtype):
    K = 4
    numel, mats = layout([(96, 200), (150, 64)], [0, 0], 65)
    cfg, plain, handle = _outer_pair(K, dtype, numel, outer_lr=2e-3, clip_threshold=0.05)
    with plain, handle, _ortho(numel, mats, "f32", scale="rms") as o:
        _settled((plain, handle), K, numel)
        # one worker flagged, the clip active
        theta, b, reps = _outer_inputs(K, dtype, numel, 1, [1e-3, 1e-3, 2e-2, 1e-3])
        st = _compare_outer(cfg, plain, handle, o, theta, b, reps, mats, "full", "flagged")
        assert st.anomalous.tolist() == [0, 0, 1, 0] and st.clip_coef < 1.0
        # a worker with a NaN
        theta, b, reps = _outer_inputs(K, dtype, numel, 2, [1e-3] * 4)
        reps[1][17] = math.nan
        st = _compare_outer(cfg, plain, handle, o, theta, b, reps, mats, "full", "nan")
        assert st.anomalous.tolist() == [0, 1, 0, 0]
        # every worker flagged: theta and b as they were (signed zeros too), replicas back to theta
        theta, b, reps = _outer_inputs(K, dtype, numel, 3, [5e-2] * 4)
        theta[5] = -0.0
        st = _compare_outer(cfg, plain, handle, o, theta, b, reps, mats, "full", "rollback")
        assert st.rolled_back
        assert math.copysign(1.0, float(theta[5])) < 0


def test_outer_step_with_no_pseudo_gradient_and_no_momentum():
    """Nothing to step along: theta stays, where normalising would divide by zero."""
    numel, mats = layout([(64, 80)], tail=3)
    theta = _randn(numel, 1, 0.02)
    b = torch.zeros(numel, device=DEV)
    reps = [theta.clone() for _ in range(3)]
    cfg = OuterConfig(3, [numel], "f32")
    with EditOuter(cfg, DEV) as h, _ortho(numel, mats, "f32") as o:
        before = theta.clone()
        h.step_layer_ortho(0, o, theta, b, reps)
        assert torch.equal(theta, before) and bool((b == 0).all())
        assert all(torch.equal(r, before) for r in reps)


def test_outer_step_without_penalty_and_without_matrices():
    """The DiLoCo weights, and a layout of no matrix: the plain outer step bit for bit."""
    numel = 3001
    cfg = OuterConfig(4, [numel], "bf16", flags=0)
    theta, b, reps = _outer_inputs(4, "bf16", numel, 9)
    t2, b2, r2 = theta.clone(), b.clone(), [r.clone() for r in reps]
    with EditOuter(cfg, DEV) as p, EditOuter(cfg, DEV) as h, _ortho(numel, [], "f32") as o:
        p.step_layer(0, theta, b, reps)
        h.step_layer_ortho(0, o, t2, b2, r2)
        torch.cuda.synchronize()
    assert torch.equal(theta, t2) and torch.equal(b, b2)
    assert all(torch.equal(x, y) for x, y in zip(reps, r2))


# ----------------------------------------------------- together, and calls


def test_local_steps_and_outer_steps_together():
    """Two rounds of three workers, two local steps each, then the outer step on
    their replicas: replayed in 64 bits from the library's state at each step."""
    K, dtype = 3, "bf16"
    numel, mats = layout([(96, 160), (160, 96)], tail=33)
    outside = ~mask_of(numel, mats, DEV)
    cfg = OuterConfig(K, [numel], dtype, outer_lr=2e-3, ema_warmup_rounds=10)
    theta, b = _randn(numel, 1, 0.02), torch.zeros(numel, device=DEV)
    reps = [theta.to(torch.bfloat16) for _ in range(K)]
    moms = [torch.zeros(numel, device=DEV) for _ in range(K)]
    with EditOuter(cfg, DEV) as plain, EditOuter(cfg, DEV) as h, \
            _ortho(numel, mats, dtype, scale="rms") as worker, _ortho(numel, mats, "f32", scale="rms") as outer:
        for rnd in range(2):
            for j in range(K):
                for step in range(2):
                    g = _randn(numel, 1000 + 100 * rnd + 10 * j + step, 1e-3).to(torch.bfloat16)
                    ref_p, ref_m, outs = _local_step64(reps[j], g, moms[j], mats, worker.cfg.scales(), 5e-3, 0.95, 0.1, True)
                    worker.local_step(reps[j], g, moms[j], lr=5e-3, mu=0.95, weight_decay=0.1)
                    _check_step(reps[j], ref_p, mats, outs, [5e-3 * s for s in worker.cfg.scales()], "fast", f"{rnd} {j} {step}")
                    reps[j][outside] -= 1e-3 * g[outside]  # the gains' own optimizer
            state = [t.clone() for t in (theta, b, *reps)]
            _compare_outer(cfg, plain, h, outer, state[0], state[1], state[2:], mats, "full", f"round {rnd}")
            h2 = EditOuter(cfg, DEV)  # the same step again, in place, from the same EMA state
            if rnd:
                st = prior
                h2.state_set(0, st.ema_mean, st.ema_std, st.round)
            h2.step_layer_ortho(0, outer, theta, b, reps)
            prior = h2.state_get(0)
            h2.close()
            assert all(torch.equal(r, theta.to(r.dtype)) for r in reps)


def test_captured_calls_replay_like_eager_ones():
    """All three calls in one HIP graph, replayed with eager work between the replays."""
    K = 3
    numel, mats = layout([(96, 200), (150, 64)], tail=5)
    cfg = OuterConfig(K, [numel], "bf16", outer_lr=2e-3)
    theta, b, reps = _outer_inputs(K, "bf16", numel, 40)
    p, g = _randn(numel, 41, 0.02).to(torch.bfloat16), _randn(numel, 42, 1e-3).to(torch.bfloat16)
    m, x = torch.zeros(numel, device=DEV), _randn(numel, 43).to(torch.bfloat16)
    out = torch.zeros_like(x)
    fixed = [theta, b, *reps, p, g, m, x, out]
    eager = [t.clone() for t in fixed]

    def calls(h, o, f, t):
        th, mo, r, (pp, gg, mm, xx, oo) = t[0], t[1], t[2:2 + K], t[2 + K:]
        o.orthogonalize(xx, oo)
        o.local_step(pp, gg, mm, lr=1e-2, weight_decay=0.1)
        h.step_layer_ortho(0, f, th, mo, r)

    with EditOuter(cfg, DEV) as ha, EditOuter(cfg, DEV) as hb, \
            _ortho(numel, mats, "bf16") as oa, _ortho(numel, mats, "bf16") as ob, \
            _ortho(numel, mats, "f32", scale="rms") as fa, _ortho(numel, mats, "f32", scale="rms") as fb:
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=torch.cuda.Stream(DEV)):
            calls(ha, oa, fa, fixed)
        torch.cuda.synchronize()
        for replay in range(4):
            for t in (g, x, *reps):
                t.add_(_randn(numel, 60 + replay, 1e-3).to(t.dtype))
            for src, dst in zip(fixed, eager):
                dst.copy_(src)
            calls(hb, ob, fb, eager)
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            for i, (a, c) in enumerate(zip(fixed, eager)):
                assert torch.equal(a, c), f"replay {replay} tensor {i}"
            assert ha.state_get(0).norm.tolist() == hb.state_get(0).norm.tolist()


def test_two_handles_on_two_streams():
    """Handles own their workspaces: calls of two of them may overlap."""
    numel, mats = layout([(512, 700), (300, 300)])
    xs = [_randn(numel, s).to(torch.bfloat16) for s in (1, 2)]
    with _ortho(numel, mats, "bf16") as a, _ortho(numel, mats, "bf16") as c:
        want = [a.orthogonalize(x) for x in xs]
        torch.cuda.synchronize()
        streams = [torch.cuda.Stream(DEV), torch.cuda.Stream(DEV)]
        got = [torch.empty_like(x) for x in xs]
        for _ in range(3):
            for h, s, x, y in zip((a, c), streams, xs, got):
                h.orthogonalize(x, y, stream=s)
        torch.cuda.synchronize()
    assert all(torch.equal(p, q) for p, q in zip(want, got))


def test_many_matrices():
    """Hundreds of matrices in one unit, some whole in a block and, beside a larger one, none."""
    shapes = [(1 + k % 13, 1 + (7 * k) % 29) for k in range(700)]
    for more in ([], [(130, 300)]):
        numel, mats = layout(shapes + more)
        x = _randn(numel, 12)
        with _ortho(numel, mats, "f32") as o:
            y = o.orthogonalize(x)
        for spec in mats[::23] + mats[-1:]:
            assert_o_close(matrix(y, spec), ortho64(matrix(x, spec)), "full", f"{spec}")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_longest_side(dtype):
    """One row, and one column, of 2^24 elements: the workspace's offsets reach 2^31 bytes and, in fp32, nearly 2^32."""
    for shape in ((1, 2 ** 24), (2 ** 24, 1)):
        x = _randn(2 ** 24, 13).to(TYPES[dtype])
        with _ortho(2 ** 24, [(0, *shape)], dtype) as o:
            y = o.orthogonalize(x)
        assert_o_close(y.view(shape), ortho64(x.view(shape)), "full" if dtype == "f32" else "fast", f"{dtype} {shape}")


def test_matrices_behind_2_to_the_31_elements():
    at = 2 ** 31 + 5
    mats = [(3, 70, 90), (at, 90, 300), (at + 90 * 300, 64, 64)]
    numel = at + 90 * 300 + 64 * 64 + 3
    x = torch.zeros(numel, dtype=torch.bfloat16, device=DEV)
    for k, spec in enumerate(mats):
        matrix(x, spec).copy_(_randn(spec[1] * spec[2], 14 + k).view(spec[1], spec[2]))
    with _ortho(numel, mats, "bf16") as o:
        y = x.clone()
        o.orthogonalize(y, y)
    for spec in mats:
        assert_o_close(matrix(y, spec), ortho64(matrix(x, spec)), "fast", f"{spec}")
        matrix(y, spec).zero_()
    assert int(y.count_nonzero()) == 0


def test_result_on_another_stream():
    """A new result belongs to the stream of the call, where memory that the
    current one has just let go, with work pending on it, is not handed out."""
    numel, mats = layout([(600, 700)])
    x = _randn(numel, 15).to(torch.bfloat16)
    side = torch.cuda.Stream(DEV)
    with _ortho(numel, mats, "bf16") as o:
        want = o.orthogonalize(x)
        torch.cuda.synchronize()
        for _ in range(3):
            held = torch.full_like(x, 2.0)
            for _ in range(20):
                held.mul_(0.5).add_(1.0)  # stays 2
            kept = held.float()
            del held
            got = o.orthogonalize(x, stream=side)
            torch.cuda.synchronize()
            assert torch.equal(got, want)
            assert bool((kept == 2.0).all())


def test_outer_step_is_timed_and_empty_units_pass():
    """Kernel times of a step with matrices, and a unit of no elements."""
    numel, mats = layout([(300, 400)], tail=9)
    cfg = OuterConfig(2, [numel, 0], "bf16")
    theta, b, reps = _outer_inputs(2, "bf16", numel, 70)
    none = torch.empty(0, device=DEV)
    with EditOuter(cfg, DEV) as h, _ortho(numel, mats, "f32", scale="rms") as o, _ortho(0, [], "f32") as empty:
        h.set_profiling(1)
        h.step_layer_ortho(0, o, theta, b, reps)
        h.step_layer_ortho(1, empty, none, none.clone(), [none.to(torch.bfloat16) for _ in range(2)])
        torch.cuda.synchronize()
        times = h.kernel_times(0)
        assert h.state_get(0).round == 1 and h.state_get(1).round == 1
    assert all(torch.equal(r, theta.to(r.dtype)) for r in reps)
    assert len(times) == 2 and min(times) > 0.0


def test_refusals():
    numel, mats = layout([(32, 40)], tail=8)
    x = _randn(numel, 1).to(torch.bfloat16)
    m = torch.zeros(numel, device=DEV)
    wide = torch.zeros(2 * numel, dtype=torch.bfloat16, device=DEV)
    with _ortho(numel, mats, "bf16") as o:
        for bad in (x.float(), x[:-1], wide[::2], x.cpu(), x.view(-1, 2).t()):
            with pytest.raises(ValueError):
                o.orthogonalize(bad)
            with pytest.raises(ValueError):
                o.local_step(x, bad, m, lr=0.1)
        with pytest.raises(TypeError):
            o.orthogonalize([1.0])
        with pytest.raises(EditOuterError, match="overlap"):
            o.orthogonalize(wide[:numel], wide[8:numel + 8])
        with pytest.raises(EditOuterError, match="aligned"):
            o.orthogonalize(wide[1:numel + 1], x.clone())
        with pytest.raises(EditOuterError, match="overlap"):
            o.local_step(x, x, m, lr=0.1)
        for kw in (dict(lr=-1.0), dict(lr=math.nan), dict(lr=0.1, mu=1.0), dict(lr=0.1, mu=-0.1), dict(lr=0.1, weight_decay=math.inf)):
            with pytest.raises(EditOuterError):
                o.local_step(x, x.clone(), m, **kw)
        reps = [torch.zeros(numel, dtype=torch.bfloat16, device=DEV)]
        theta, b = torch.zeros(numel, device=DEV), torch.zeros(numel, device=DEV)
        with EditOuter(OuterConfig(1, [numel, numel + 1], "bf16"), DEV) as h:
            with pytest.raises(TypeError):
                h.step_layer_ortho(0, None, theta, b, reps)
            with pytest.raises(IndexError):
                h.step_layer_ortho(2, o, theta, b, reps)
            with pytest.raises(EditOuterError, match="unit has"):
                h.step_layer_ortho(1, o, torch.zeros(numel + 1, device=DEV), torch.zeros(numel + 1, device=DEV),
                                   [torch.zeros(numel + 1, dtype=torch.bfloat16, device=DEV)])
            with pytest.raises(EditOuterError, match="overlap"):
                h.step_layer_ortho(0, o, theta, theta, reps)
        with EditOuter(OuterConfig(1, [numel], "bf16", flags=ONE_PASS), DEV) as h:
            with pytest.raises(EditOuterError, match="ONE_PASS"):
                h.step_layer_ortho(0, o, theta, b, reps)
    assert AE | WA | GC == 7 and DEFAULT[0] == 3.4445
