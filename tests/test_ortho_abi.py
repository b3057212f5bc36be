"""CPU-side checks of the orthogonalised updates: the ABI's names and
structures, and what edit_ortho_init and the binding refuse before a GPU is
touched."""
import ctypes
import math
import os
import re

import pytest
import torch

from paper_2412_07210_amd import OrthoConfig, Orthogonalizer, outer
from ortho_reference import DEFAULT, ortho64

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_header_declarations_match_binding():
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "edit_outer.h")).read(), flags=re.S)
    assert sorted(set(re.findall(r"\b(edit_ortho_\w+)\s*\(", text))) == sorted(outer.ORTHO_EXPORTS)
    lib = outer.load_library()
    for name in outer.ORTHO_EXPORTS:
        assert hasattr(lib, name), name


def test_struct_layouts():
    assert ctypes.sizeof(outer._OrthoMatrix) == 8 + 4 + 4 + 8
    assert ctypes.sizeof(outer._OrthoConfig) == 8 + 8 + 4 * 4 + 8
    assert outer._OrthoConfig.coefficients.offset == 32


def _init(numel=64, matrices=((0, 8, 8, 1.0),), coefficients=None, null_matrices=False, **over):
    lib = outer.load_library()
    arr = (outer._OrthoMatrix * max(1, len(matrices)))(*[outer._OrthoMatrix(*m) for m in matrices])
    fields = dict(numel=numel, matrices=arr, num_matrices=len(matrices), dtype=1, precision=0, steps=5)
    fields.update(over)
    if null_matrices:
        fields.pop("matrices")
    if coefficients is not None:
        fields["coefficients"] = (ctypes.c_double * len(coefficients))(*coefficients)
    cfg = outer._OrthoConfig(**fields)
    h = ctypes.c_void_p(1)
    rc = lib.edit_ortho_init(ctypes.byref(cfg), ctypes.byref(h))
    assert not h.value
    return rc, lib.edit_outer_last_error().decode()


BIG = 2 ** 40


@pytest.mark.parametrize("over,needle", [
    (dict(numel=-1, matrices=()), "numel"),
    (dict(num_matrices=-1), "num_matrices"),
    (dict(null_matrices=True), "matrices must not be NULL"),
    (dict(dtype=2), "dtype"),
    (dict(precision=2), "precision"),
    (dict(precision=-1), "precision"),
    (dict(steps=0), "steps"),
    (dict(steps=33), "steps"),
    (dict(matrices=((0, -1, 8, 1.0),)), "rows and cols"),
    (dict(matrices=((0, 8, -8, 1.0),)), "rows and cols"),
    (dict(matrices=((-1, 8, 4, 1.0),)), "beyond the unit"),
    (dict(matrices=((1, 8, 8, 1.0),)), "beyond the unit"),
    (dict(matrices=((65, 0, 8, 1.0),)), "beyond the unit"),
    (dict(matrices=((2 ** 62, 8, 8, 1.0),)), "beyond the unit"),
    (dict(matrices=((0, 4, 8, 1.0), (31, 4, 8, 1.0))), "overlap"),
    (dict(matrices=((32, 4, 8, 1.0), (0, 4, 9, 1.0))), "overlap"),
    (dict(matrices=((0, 8, 8, math.nan),)), "scale"),
    (dict(matrices=((0, 8, 8, math.inf),)), "scale"),
    (dict(numel=BIG, matrices=((0, 2 ** 24 + 1, 1, 1.0),)), "2^24"),
    (dict(numel=BIG, matrices=((0, 2 ** 15 + 1, 2 ** 14, 1.0),)), "too large"),
    (dict(numel=BIG, matrices=((0, 2 ** 31 - 1, 2 ** 31 - 1, 1.0),)), "2^24"),
    (dict(steps=1, coefficients=(math.nan, 0, 0)), "finite"),
    (dict(steps=2, coefficients=(1, 0, 0, 1, math.inf, 0)), "step 1"),
    (dict(steps=1, coefficients=(4.5, 0, 0)), "beyond 4"),
    (dict(steps=1, coefficients=(20, -40, 20)), "exceeds 15"),
    (dict(steps=2, coefficients=(2, 0, 0, 2.5, 0, 0)), "step 1"),
])
def test_init_refuses(over, needle):
    rc, msg = _init(**over)
    assert rc == outer.EDIT_EINVAL
    assert needle in msg


@pytest.mark.skipif(torch.cuda.is_available(), reason="the CPU's answer to a good configuration")
@pytest.mark.parametrize("over", [
    dict(),
    dict(matrices=()),
    dict(numel=0, matrices=()),
    dict(matrices=((64, 0, 8, 1.0), (3, 5, 0, 0.0))),
    dict(matrices=((0, 4, 8, 1.0), (32, 8, 4, -1.0))),
    dict(steps=1, coefficients=(8.2, -23.0, 16.8)),
    dict(numel=2 ** 29, matrices=((0, 2 ** 15, 2 ** 14, 1.0),)),
    dict(numel=BIG, matrices=((0, 32, 2 ** 24, 1.0),)),
])
def test_init_accepts_up_to_the_device(over):
    rc, msg = _init(**over)
    assert rc in (outer.EDIT_ENODEV, outer.EDIT_EHIP)


def test_null_arguments():
    lib = outer.load_library()
    h = ctypes.c_void_p()
    assert lib.edit_ortho_init(None, ctypes.byref(h)) == outer.EDIT_EINVAL
    cfg = outer._OrthoConfig()
    assert lib.edit_ortho_init(ctypes.byref(cfg), None) == outer.EDIT_EINVAL
    assert lib.edit_ortho_apply(None, None, None, None) == outer.EDIT_EINVAL
    assert lib.edit_ortho_local_step(None, None, None, None, 0.1, 0.9, 0.0, 1, None) == outer.EDIT_EINVAL
    ptrs = (ctypes.c_void_p * 1)()
    assert lib.edit_outer_step_layer_ortho(None, 0, None, None, None, ptrs, None) == outer.EDIT_EINVAL
    lib.edit_ortho_destroy(None)


@pytest.mark.parametrize("over,error", [
    (dict(dtype="f16"), "dtype"),
    (dict(precision="half"), "precision"),
    (dict(scale="adam"), "scale"),
    (dict(scale=[1.0, 2.0]), "scales"),
    (dict(coefficients=[1.0, 2.0]), "coefficients"),
    (dict(coefficients=[[1.0, 2.0, 0.0]] * 3), "coefficients"),
    (dict(matrices=[(0, 2.5, 4)]), "whole numbers"),
    (dict(matrices=[(0, 2 ** 32 + 8, 8)]), "2\\^31"),
])
def test_binding_refuses(over, error):
    cfg = OrthoConfig(**{**dict(numel=64, matrices=[(0, 8, 8)]), **over})
    with pytest.raises(ValueError, match=error):
        Orthogonalizer(cfg, "cuda:0")


def test_binding_needs_a_gpu_device():
    with pytest.raises(ValueError, match="GPU device"):
        Orthogonalizer(OrthoConfig(64, [(0, 8, 8)]), "cpu")


def test_scales_and_precision_defaults():
    m = [(0, 8, 8), (64, 32, 2), (128, 2, 32)]
    assert OrthoConfig(192, m).scales() == [1.0, 4.0, 1.0]
    assert OrthoConfig(192, m, scale="rms").scales() == pytest.approx([0.2 * math.sqrt(x) for x in (8, 32, 32)])
    assert OrthoConfig(192, m, scale=[1, 2, 3]).scales() == [1.0, 2.0, 3.0]
    assert OrthoConfig(0, [(0, 0, 4)]).scales() == [0.0]
    for dtype, precision, want in (("bf16", None, 0), ("f32", None, 1), ("f32", "fast", 0), ("bf16", "full", 1)):
        c, _ = Orthogonalizer._c_config(OrthoConfig(192, m, dtype=dtype, precision=precision))
        assert c.precision == want


def test_reference_brings_singular_values_near_one():
    """The reference itself: singular vectors kept, singular values through the scalar iteration."""
    gen = torch.Generator().manual_seed(3)
    for rows, cols in ((12, 12), (9, 20), (20, 9)):
        u = torch.randn(rows, cols, generator=gen, dtype=torch.float64)
        left, s, right = torch.linalg.svd(u, full_matrices=False)
        s = s / u.norm()
        for _ in range(5):
            s = DEFAULT[0] * s + DEFAULT[1] * s ** 3 + DEFAULT[2] * s ** 5
        assert torch.allclose(ortho64(u), left @ torch.diag(s) @ right, atol=1e-10)
        assert float(s.min()) > 0.3 and float(s.max()) < 1.3
