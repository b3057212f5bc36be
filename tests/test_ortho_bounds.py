"""The error bound of orthogonalised updates, on the CPU: the emulated
arithmetic stays within it, and an iteration that loses X's low half does not
where the matrix lacks directions."""
import pytest
import torch

from ortho_emulation import emulate, reference_and_bound

GENERAL = [(2, 2), (4, 4), (8, 8), (8, 300), (16, 16), (16, 200), (200, 16), (64, 64), (100, 200), (128, 128), (200, 170)]


def spectrum(kind, rows, cols, seed):
    g = torch.Generator().manual_seed(seed)
    if kind == "gauss":
        return torch.randn(rows, cols, generator=g)
    if kind == "same":
        return torch.ones(rows, cols)
    if kind == "one":
        out = torch.zeros(rows, cols)
        out[rows // 2, cols // 3] = -3.0
        return out
    rank = int(kind[4:])
    return torch.randn(rows, rank, generator=g) @ torch.randn(rank, cols, generator=g)


def error(o, ref):
    return float((o.double() - ref).norm() / ref.norm())


@pytest.mark.parametrize("precision", ["fast", "full"])
@pytest.mark.parametrize("kind", ["gauss", "rank1", "rank2", "rank4", "rank16", "one", "same"])
def test_emulated_arithmetic_stays_within_the_bound(kind, precision):
    for rows, cols in GENERAL:
        if kind.startswith("rank") and int(kind[4:]) >= min(rows, cols):
            continue
        for seed in range(3):
            u = spectrum(kind, rows, cols, seed)
            ref, bound = reference_and_bound(u, precision, deficient=kind != "gauss", alike=kind in ("one", "same"))
            off = error(emulate(u, precision), ref)
            assert off <= bound, f"{rows}x{cols} seed {seed}: {off:.3g}, bound {bound:.3g}"


@pytest.mark.parametrize("kind", ["rank1", "rank4", "rank16"])
@pytest.mark.parametrize("rows,cols", [(128, 128), (100, 200), (60, 250), (200, 170), (300, 700), (600, 600)])
def test_a_lost_low_half_breaks_the_bound(kind, rows, cols):
    u = spectrum(kind, rows, cols, 1)
    ref, bound = reference_and_bound(u, "fast", deficient=True)
    assert error(emulate(u, "fast"), ref) <= bound
    assert error(emulate(u, "fast", low=False), ref) > bound


@pytest.mark.parametrize("steps", [3, 4, 6, 8])
def test_a_lost_low_half_breaks_the_bound_at_other_step_counts(steps):
    for rows, cols in ((128, 128), (200, 170)):
        u = spectrum("rank1", rows, cols, 2)
        ref, bound = reference_and_bound(u, "fast", steps=steps, deficient=True)
        assert error(emulate(u, "fast", steps=steps), ref) <= bound
        assert error(emulate(u, "fast", steps=steps, low=False), ref) > bound


def test_steep_polynomials_stay_within_the_bound():
    """Polynomials that pass a singular value's error on 174 times."""
    coef = [(8.29, -23.6, 17.3), (4.1, -2.95, 0.545), (3.9, -2.9, 0.55)]
    for rows, cols in ((128, 128), (150, 260), (40, 90)):
        for seed in range(6):
            u = spectrum("rank1", rows, cols, seed)
            ref, bound = reference_and_bound(u, "fast", steps=3, coefficients=coef, deficient=True, rank_one=True, counted=9)
            off = error(emulate(u, "fast", steps=3, coefficients=coef), ref)
            assert off <= bound < 0.3, f"{rows}x{cols} seed {seed}: {off:.3g}, bound {bound:.3g}"
