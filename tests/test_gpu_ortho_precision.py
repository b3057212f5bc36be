"""Errors of the orthogonalised updates on updates that lack directions, for
every kernel that FAST is dispatched to, for other step counts, and for steps
of parameters (GPU).  The bounds are derived in ortho_emulation.py; an
iteration that loses the low half of X exceeds them (test_ortho_bounds.py).
Handles are fp32, so that no output rounding covers an error."""
import math

import pytest
import torch

from ortho_emulation import reference_and_bound
from ortho_reference import half_step, layout, matrix
from paper_2412_07210_amd import EditOuter, OrthoConfig, Orthogonalizer, OuterConfig

pytestmark = pytest.mark.gpu

DEV = torch.device("cuda:0")
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def _randn(rows, cols, seed, std=1.0):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    return torch.empty(rows, cols, device=DEV).normal_(0.0, std, generator=gen)


def _of_rank(rank, rows, cols, seed):
    return _randn(rows, rank, seed) @ _randn(rank, cols, seed + 1)


def _orthogonalize(shape, u, precision, **more):
    rows, cols = shape
    with Orthogonalizer(OrthoConfig(rows * cols, [(0, rows, cols)], dtype="f32", precision=precision, **more), DEV) as o:
        return o.orthogonalize(u.reshape(-1)).view(rows, cols)


def _error(o, ref):
    return float((o.double() - ref).norm() / ref.norm())


# The kernels that a shape's products run in with FAST (256 CUs).
DISPATCHES = {
    "one block, 32 wide": (24, 200),
    "one block, 64 wide": (250, 60),
    "one block, 128 wide": (128, 128),
    "one block, 128 wide, ragged": (100, 200),
    "tiles of 64, four slabs": (300, 260),
    "tiles of 64, two slabs (update)": (900, 3900),
    "tiles of 64, two slabs (symmetric), update of 128": (2100, 2120),
    "tiles of 128": (3700, 3600),
    "update of 256": (500, 29201),
    "update of 256, tall": (29192, 504),
}


@pytest.mark.parametrize("rank", [1, 4, 16])
@pytest.mark.parametrize("kernels", DISPATCHES)
def test_updates_that_lack_directions(kernels, rank):
    shape = DISPATCHES[kernels]
    u = _of_rank(rank, *shape, 40 + rank)
    for precision in ("fast", "full"):
        ref, bound = reference_and_bound(u, precision, deficient=True)
        off = _error(_orthogonalize(shape, u, precision), ref)
        assert off <= bound + half_step(torch.float32), f"{precision} {kernels}: {off:.3g}, bound {bound:.3g}"


def _documented(precision, r, whole):
    """What the header says that O is off by at most, of its norm."""
    if precision == "full":
        return 6e-6 if whole else 2.5e-4
    if r < 64:
        return 0.25 / r
    return 1.3e-3 if whole else 5e-3


@pytest.mark.parametrize("precision", ["fast", "full"])
@pytest.mark.parametrize("shape", [(2, 2), (4, 4), (8, 8), (8, 3000), (16, 16), (200, 16), (32, 32), (64, 64), (64, 300),
                                   (128, 128), (512, 512), (700, 1024), (1024, 1024)], ids=lambda s: "%dx%d" % s)
def test_documented_errors(shape, precision):
    r = min(shape)
    for seed in range(3):
        for rank in (1, 2, 4, 16, r):
            if rank > r:
                continue
            u = _of_rank(rank, *shape, seed) if rank < r else _randn(*shape, seed)
            ref, _ = reference_and_bound(u, precision)
            off = _error(_orthogonalize(shape, u, precision), ref)
            assert off <= _documented(precision, r, rank == r), f"{precision} {shape} rank {rank} seed {seed}: {off:.3g}"
    if precision == "fast":
        one = torch.zeros(shape, device=DEV)
        one[shape[0] // 2, shape[1] // 3] = -3.0
        for u in (torch.ones(shape, device=DEV), one):  # elements that round alike
            ref, _ = reference_and_bound(u, precision)
            assert _error(_orthogonalize(shape, u, precision), ref) <= 2.5e-2


@pytest.mark.parametrize("shape", [(64, 64), (1024, 1024), (2048, 5632), (4096, 4096)], ids=lambda s: "%dx%d" % s)
def test_documented_errors_of_layers(shape):
    """Full, nearly low and low rank up to a layer's sizes."""
    r = min(shape)
    nearly = _of_rank(16, *shape, 81) + 0.1 * _randn(*shape, 83)
    full = 2.4e-4 + 1.3e-5 * math.sqrt(r)  # above the derived bound for every rank
    cases = [(_randn(*shape, 80), 2e-3, 6e-6), (nearly, 2e-3, full)]
    for rank in (1, 4, 16):
        u = _of_rank(rank, *shape, 84)
        assert reference_and_bound(u, "full", deficient=True)[1] <= full
        cases.append((u, 5e-3, full))
    for u, *documented in cases:
        ref, _ = reference_and_bound(u, "full")
        for precision, most in zip(("fast", "full"), documented):
            off = _error(_orthogonalize(shape, u, precision), ref)
            assert off <= most, f"{precision} {shape}: {off:.3g}, documented {most:.3g}"


@pytest.mark.parametrize("steps", [1, 2, 3, 4, 6, 8])
@pytest.mark.parametrize("shape", [(128, 128), (200, 170), (900, 3900), (2100, 2120), (500, 29201)], ids=lambda s: "%dx%d" % s)
def test_fast_at_other_step_counts(shape, steps):
    """Which buffer holds X, which steps write its low half and which read it."""
    for rank in (1, None):
        u = _randn(*shape, 50) if rank is None else _of_rank(rank, *shape, 50)
        ref, bound = reference_and_bound(u, "fast", steps=steps, deficient=rank is not None)
        off = _error(_orthogonalize(shape, u, "fast", steps=steps), ref)
        assert off <= bound + half_step(torch.float32), f"rank {rank} {steps} steps: {off:.3g}, bound {bound:.3g}"


@pytest.mark.parametrize("shape", [(128, 128), (150, 260), (2100, 2120)], ids=lambda s: "%dx%d" % s)
@pytest.mark.parametrize("coef", [
    [(1.5, -0.5, 0.0)] * 4,
    [(3.4445, -4.7750, 2.0315), (1.5, -0.5, 0.0), (3.4445, -4.7750, 2.0315), (2.0, -1.5, 0.5)],
    [(8.29, -23.6, 17.3), (4.1, -2.95, 0.545), (3.9, -2.9, 0.55)],
], ids=["cubic", "mixed", "steep"])
def test_fast_with_coefficients_of_each_step(shape, coef):
    # the steep polynomials reach 8.3, three times the default's: three steps count as nine
    counted = 9 if len(coef) == 3 else len(coef)
    for rank in (1, None):
        u = _randn(*shape, 51) if rank is None else _of_rank(rank, *shape, 51)
        ref, bound = reference_and_bound(u, "fast", steps=len(coef), coefficients=coef, deficient=rank is not None,
                                         rank_one=rank == 1, counted=counted)
        off = _error(_orthogonalize(shape, u, "fast", steps=len(coef), coefficients=coef), ref)
        assert off <= bound + half_step(torch.float32), f"rank {rank}: {off:.3g}, bound {bound:.3g}"


# ------------------------------------------------------------ steps of parameters


def _step_error(got, ref, mats, outs, factors, bounds, what):
    """2-norm of each matrix's error against its step's: the bound of O, and one rounding of the result."""
    for spec, o, f, bound in zip(mats, outs, factors, bounds):
        y, e = matrix(got, spec).double(), matrix(ref, spec)
        step = f * float(o.norm())
        off, allowed = float((y - e).norm()), bound * step + half_step(got.dtype) * float(e.norm())
        assert off <= allowed * (1 + 1e-6), f"{what} {spec}: {off / step:.3g} of the step, allowed {allowed / step:.3g}"


@pytest.mark.parametrize("precision", ["fast", "full"])
@pytest.mark.parametrize("shapes", [[(128, 128), (60, 250)], [(96, 200), (300, 64), (77, 77)], [(2100, 2120)], [(500, 29201)]],
                         ids=["one block", "tiles of 64", "tiles of 128", "update of 256"])
def test_error_of_a_local_step(shapes, precision):
    lr, mu, decay = 0.02, 0.9, 0.1
    numel, mats = layout(shapes)
    p, m = _randn(1, numel, 60, 0.02).view(-1), _randn(1, numel, 61, 1e-3).view(-1)
    g = _randn(1, numel, 62, 1e-3).view(-1)
    ref, outs, bounds = p.double(), [], []
    with Orthogonalizer(OrthoConfig(numel, mats, dtype="f32", precision=precision, scale="rms"), DEV) as o:
        factors = [lr * s for s in o.cfg.scales()]
        for spec, f in zip(mats, factors):
            gg, mm, pp = matrix(g, spec).double(), matrix(m, spec).double(), matrix(ref, spec)
            out, bound = reference_and_bound(gg + mu * (mu * mm + gg), precision)
            pp.mul_(1 - lr * decay).sub_(f * out)
            outs.append(out), bounds.append(bound)
        o.local_step(p, g, m, lr=lr, mu=mu, weight_decay=decay)
    _step_error(p, ref, mats, outs, factors, bounds, precision)


@pytest.mark.parametrize("precision", ["full", "fast"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("shapes", [[(96, 200), (300, 64), (77, 77)], [(1300, 1290)], [(2100, 2120), (90, 70)], [(500, 29201)]],
                         ids=["small", "tiles of 64", "tiles of 128", "update of 256"])
def test_error_of_an_outer_step(shapes, dtype, precision):
    """Theta, the momentum and the replicas of either type, at every tile side of the last product."""
    K, nu, rho = 3, 2e-3, 0.85
    numel, mats = layout(shapes, gaps=[5] + [0] * (len(shapes) - 1), tail=11)
    theta, b = _randn(1, numel, 70, 0.02).view(-1), _randn(1, numel, 71, 1e-3).view(-1)
    reps = [(theta + _randn(1, numel, 72 + j, 1e-3 * (1 + 0.1 * j)).view(-1)).to(TYPES[dtype]) for j in range(K)]
    cfg = OuterConfig(K, [numel], dtype, outer_lr=nu, momentum=rho)
    old, b0 = theta.double(), b.double()
    gaps = [r.clone() for r in reps]
    with EditOuter(cfg, DEV) as h, Orthogonalizer(
            OrthoConfig(numel, mats, dtype="f32", precision=precision, scale="rms"), DEV) as o:
        factors = [nu * s for s in o.cfg.scales()]
        h.step_layer_ortho(0, o, theta, b, reps)
        st = h.state_get(0)
    d = sum(st.clip_coef * w * (r.double() - old) for w, r in zip(st.weight, gaps))
    want = rho * b0 - d
    # one rounding, and D's own in 64 bits (the weights are the library's)
    assert bool(((b.double() - want).abs() <= half_step(torch.float32) * want.abs() * (1 + 1e-6) + 1e-16).all())
    u = rho * want - d
    ref, outs, bounds = old - nu * u, [], []
    for spec, f in zip(mats, factors):
        out, bound = reference_and_bound(matrix(u, spec), precision)
        matrix(ref, spec).copy_(matrix(old, spec) - f * out)
        outs.append(out), bounds.append(bound)
    _step_error(theta, ref, mats, outs, factors, bounds, f"{dtype} {precision}")
    outside = torch.ones(numel, dtype=torch.bool, device=DEV)
    for at, rows, cols in mats:
        outside[at:at + rows * cols] = False
    off = (theta.double() - ref).abs()[outside]
    assert bool((off <= half_step(torch.float32) * ref.abs()[outside] * (1 + 1e-6) + 1e-16).all())
    assert all(torch.equal(r, theta.to(r.dtype)) for r in reps)
    assert math.isfinite(st.synced_norm)
