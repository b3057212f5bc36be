"""What the binding of the orthogonalised updates refuses beside
test_ortho_abi.py: numbers that the C structures would cut off (CPU)."""
import math

import pytest

from paper_2412_07210_amd import OrthoConfig, Orthogonalizer


@pytest.mark.parametrize("over,error", [
    (dict(numel=2 ** 64 + 64), "numel"),
    (dict(numel=2 ** 63), "numel"),
    (dict(numel=64.5), "numel"),
    (dict(matrices=[(2 ** 64, 8, 8)]), "offset"),
    (dict(matrices=[(-2 ** 64, 8, 8)]), "offset"),
    (dict(matrices=[(0.5, 8, 8)]), "whole numbers"),
    (dict(matrices=[(0, 8)]), "offset, rows, cols"),
    (dict(steps=2 ** 32 + 5), "steps"),
    (dict(steps=2.5), "steps"),
    (dict(steps=2.5, coefficients=[1.0, 0.0, 0.0]), "steps"),
])
def test_numbers_that_would_be_cut_off(over, error):
    """2^64 + 64 elements would become 64, an offset of 2^64 the unit's start, 2.5 steps two."""
    cfg = OrthoConfig(**{**dict(numel=64, matrices=[(0, 8, 8)]), **over})
    with pytest.raises(ValueError, match=error):
        Orthogonalizer._c_config(cfg)


def test_numbers_arrive_as_given():
    m = [(2 ** 62, 3, 5), (7, 2 ** 24, 32)]
    c, _ = Orthogonalizer._c_config(OrthoConfig(2 ** 63 - 1, m, steps=32, scale=[0.5, -2.0]))
    assert c.numel == 2 ** 63 - 1 and c.steps == 32 and c.num_matrices == 2
    assert [(c.matrices[i].offset, c.matrices[i].rows, c.matrices[i].cols) for i in range(2)] == m
    assert [c.matrices[i].scale for i in range(2)] == [0.5, -2.0]
    c, _ = Orthogonalizer._c_config(OrthoConfig(64.0, [(0, 8.0, 8)], steps=2.0, coefficients=[1.5, -0.5, 0.0]))
    assert c.numel == 64 and c.steps == 2 and c.matrices[0].rows == 8
    assert [c.coefficients[k] for k in range(6)] == [1.5, -0.5, 0.0] * 2
    assert math.isclose(c.matrices[0].scale, 1.0)
