"""CPU-side checks of the AdamW step: the ABI's names and structures, what is
refused before a GPU is touched, and the reference that the GPU tests use."""
import ctypes
import math
import os
import re
import shutil
import subprocess

import numpy as np
import pytest
import torch

import adamw_reference as ref
from paper_2412_07210_amd import AdamW, AdamWConfig, AdamWState, outer

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_header_declarations_match_binding():
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "edit_outer.h")).read(), flags=re.S)
    assert sorted(set(re.findall(r"\b(edit_adamw_\w+)\s*\(", text))) == sorted(outer.ADAMW_EXPORTS)
    lib = outer.load_library()
    for name in outer.ADAMW_EXPORTS:
        assert hasattr(lib, name), name


def test_header_layout_matches_binding(tmp_path):
    """A C program of the header says every structure's size and offsets, and the constants."""
    cc = shutil.which("gcc") or shutil.which("cc")
    if cc is None:
        pytest.skip("no C compiler")
    structs = {"edit_adamw_config_t": outer._AdamWConfig, "edit_adamw_tensors_t": outer._AdamWTensors,
               "edit_adamw_call_t": outer._AdamWCall, "edit_adamw_state_t": outer._AdamWState}
    consts = {"EDIT_ADAMW_F32": outer.ADAMW_F32, "EDIT_ADAMW_E4M3": outer.ADAMW_E4M3, "EDIT_ADAMW_BLOCK": outer.ADAMW_BLOCK,
              "EDIT_ADAMW_STOCHASTIC": outer.ADAMW_STOCHASTIC}
    lines = ["#include <stddef.h>", "#include <stdio.h>", '#include "edit_outer.h"', "int main(void) {"]
    for c, s in structs.items():
        lines.append(f'  printf("{c} %zu\\n", sizeof({c}));')
        lines += [f'  printf("{c}.{f} %zu\\n", offsetof({c}, {f}));' for f, _ in s._fields_]
    lines += [f'  printf("{c} %ld\\n", (long)({c}));' for c in consts] + ["  return 0;", "}"]
    src = tmp_path / "layout.c"
    src.write_text("\n".join(lines) + "\n")
    subprocess.run([cc, "-std=c11", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(tmp_path / "layout")], check=True)
    got = dict(x.split() for x in subprocess.run([str(tmp_path / "layout")], check=True, capture_output=True,
                                                 text=True).stdout.splitlines())
    for c, s in structs.items():
        assert int(got[c]) == ctypes.sizeof(s), c
        for f, _ in s._fields_:
            assert int(got[f"{c}.{f}"]) == getattr(s, f).offset, f"{c}.{f}"
    for c, value in consts.items():
        assert int(got[c]) == value, c


def _init(numel=(64, 8), decay=None, null_numel=False, **over):
    lib = outer.load_library()
    fields = dict(num_tensors=len(numel), numel=(ctypes.c_int64 * max(1, len(numel)))(*numel), dtype=1, grad_dtype=1, held=0,
                  flags=0, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.1)
    if decay is not None:
        fields["decay"] = (ctypes.c_double * len(decay))(*decay)
    fields.update(over)
    if null_numel:
        fields.pop("numel")
    cfg = outer._AdamWConfig(**fields)
    h = ctypes.c_void_p(1)
    rc = lib.edit_adamw_init(ctypes.byref(cfg), ctypes.byref(h))
    return rc, lib.edit_outer_last_error().decode(), h


@pytest.mark.parametrize("over,needle", [
    (dict(num_tensors=-1), "num_tensors"),
    (dict(null_numel=True), "numel must not be NULL"),
    (dict(numel=(3, -1)), "numel[1] is negative"),
    (dict(numel=(2 ** 33 + 1,)), "2^33"),
    (dict(dtype=2), "dtype"),
    (dict(grad_dtype=-1), "grad_dtype"),
    (dict(held=2), "held"),
    (dict(held=-1), "held"),
    (dict(flags=2), "flag"),
    (dict(flags=1, dtype=0), "bf16"),
    (dict(beta1=1.0), "beta1"),
    (dict(beta1=-0.1), "beta1"),
    (dict(beta1=math.nan), "beta1"),
    (dict(beta2=1.0), "beta2"),
    (dict(beta2=math.inf), "beta2"),
    (dict(eps=0.0), "eps"),
    (dict(eps=1e-13), "eps"),
    (dict(eps=math.nan), "eps"),
    (dict(eps=math.inf), "eps"),
    (dict(weight_decay=-1e-9), "weight_decay"),
    (dict(weight_decay=math.inf), "weight_decay"),
    (dict(decay=(1.0, -1.0)), "decay[1]"),
    (dict(decay=(math.nan, 1.0)), "decay[0]"),
])
def test_init_refuses(over, needle):
    rc, msg, h = _init(**over)
    assert rc == outer.EDIT_EINVAL and not h.value
    assert needle in msg


@pytest.mark.skipif(torch.cuda.is_available(), reason="the CPU's answer to a good configuration")
@pytest.mark.parametrize("over", [
    dict(), dict(numel=()), dict(numel=(), null_numel=True), dict(numel=(0, 0, 5)), dict(numel=(2 ** 33,)),
    dict(dtype=0, grad_dtype=1, held=1), dict(flags=1), dict(beta1=0.0, beta2=0.0), dict(eps=1e-12),
    dict(decay=(0.0, 2.5)),
])
def test_init_accepts_up_to_the_device(over):
    rc, msg, h = _init(**over)
    assert rc in (outer.EDIT_ENODEV, outer.EDIT_EHIP) and not h.value


def test_null_arguments():
    lib = outer.load_library()
    h = ctypes.c_void_p()
    cfg, tensors, call, state = outer._AdamWConfig(), outer._AdamWTensors(), outer._AdamWCall(), outer._AdamWState()
    assert lib.edit_adamw_init(None, ctypes.byref(h)) == outer.EDIT_EINVAL
    assert lib.edit_adamw_init(ctypes.byref(cfg), None) == outer.EDIT_EINVAL
    assert lib.edit_adamw_sumsq(None, None, None, None) == outer.EDIT_EINVAL
    assert lib.edit_adamw_step(None, ctypes.byref(tensors), ctypes.byref(call), None) == outer.EDIT_EINVAL
    assert lib.edit_adamw_pack(None, None, None, ctypes.byref(tensors), 0, None) == outer.EDIT_EINVAL
    assert lib.edit_adamw_unpack(None, ctypes.byref(tensors), None, None, None) == outer.EDIT_EINVAL
    assert lib.edit_adamw_state_get(None, ctypes.byref(state)) == outer.EDIT_EINVAL
    assert lib.edit_adamw_state_set(None, 0) == outer.EDIT_EINVAL
    lib.edit_adamw_destroy(None)


@pytest.mark.parametrize("over,error", [
    (dict(dtype="f16"), "dtype"),
    (dict(grad_dtype="f64"), "grad_dtype"),
    (dict(state="8bit"), "state"),
    (dict(betas=(0.9,)), "betas"),
    (dict(numel=[64.5]), "numel"),
    (dict(numel=[2 ** 63]), "numel"),
    (dict(decay=[1.0, 1.0]), "decay"),
])
def test_binding_refuses(over, error):
    with pytest.raises(ValueError, match=error):
        AdamW(AdamWConfig(**{**dict(numel=[64]), **over}), "cuda:0")


def test_binding_needs_a_gpu_device():
    with pytest.raises(ValueError, match="GPU device"):
        AdamW(AdamWConfig([64]), "cpu")


def _bare(**over):
    """A handle's binding without its handle: what it checks by itself, with CPU tensors."""
    cfg = AdamWConfig(**{**dict(numel=[300, 0, 7], dtype="f32"), **over})
    o = AdamW.__new__(AdamW)
    o.cfg, o.device, o._h = cfg, torch.device("cpu"), None
    o._numel, o._held = list(cfg.numel), cfg.state == "e4m3"
    o._dtype = o._grad_dtype = torch.float32
    return o


def test_binding_checks_tensors():
    o = _bare()
    good = [torch.zeros(n) for n in o._numel]
    state = o.new_state()
    o.prepare(good, good, state)
    o.prepare(good, [None, None, good[2]], state)
    with pytest.raises(TypeError, match="params"):
        o.prepare([None, *good[1:]], good, state)
    with pytest.raises(ValueError, match="expected 3 tensors"):
        o.prepare(good[:2], good, state)
    for bad in (torch.zeros(299), torch.zeros(300, dtype=torch.bfloat16), torch.zeros(600)[::2]):
        with pytest.raises(ValueError, match=r"grads\[0\]"):
            o.prepare(good, [bad, *good[1:]], state)
    with pytest.raises(TypeError, match="AdamWState"):
        o.prepare(good, good, None)
    with pytest.raises(ValueError, match="no scales"):
        o.prepare(good, good, AdamWState(state.exp_avg, state.exp_avg_sq, good, good))
    e = _bare(state="e4m3")
    held = e.new_state()
    e.prepare(good, good, held)
    with pytest.raises(ValueError, match="exp_avg"):
        e.prepare(good, good, state)
    with pytest.raises(ValueError, match="missing"):
        e.prepare(good, good, AdamWState(held.exp_avg, held.exp_avg_sq, held.exp_avg_scale))
    with pytest.raises(ValueError, match="exp_avg_sq_scale"):
        e.prepare(good, good, AdamWState(held.exp_avg, held.exp_avg_sq, held.exp_avg_scale, good))


@pytest.mark.parametrize("more,error", [
    (dict(max_norm=0.0), "max_norm"), (dict(max_norm=-1.0), "max_norm"), (dict(max_norm=math.inf), "max_norm"),
    (dict(max_norm=math.nan), "max_norm"), (dict(seed=-1), "seed"), (dict(seed=2 ** 64), "seed"), (dict(seed=0.5), "seed"),
    (dict(lr=torch.zeros(1)), "lr"), (dict(lr=torch.zeros(2, dtype=torch.float64)), "lr"),
    (dict(sumsq=torch.zeros(1)), "sumsq"),
])
def test_run_refuses(more, error):
    o = _bare()
    good = [torch.zeros(n) for n in o._numel]
    plan = o.prepare(good, good, o.new_state())
    with pytest.raises(ValueError, match=error):
        plan.run(**{**dict(lr=1e-3), **more})


def test_new_state_layout():
    o = _bare(numel=[300, 1, 256, 0, 513], state="e4m3")
    s = o.new_state()
    for x in (s.exp_avg, s.exp_avg_sq):
        assert [t.numel() for t in x] == [300, 1, 256, 0, 513]
        assert all(t.dtype == torch.float8_e4m3fn for t in x)
        assert [t.data_ptr() - x[0].data_ptr() for t in x][:3] == [0, 512, 768]
        assert x[4].data_ptr() - x[0].data_ptr() == 1024
    for x in (s.exp_avg_scale, s.exp_avg_sq_scale):
        assert [t.numel() for t in x] == [2, 1, 1, 0, 3]
    s = _bare(numel=[300, 1]).new_state()
    assert [t.numel() for t in s.exp_avg] == [300, 1] and s.exp_avg_scale is None
    assert s.exp_avg[1].data_ptr() - s.exp_avg[0].data_ptr() == 4 * 512


# ---- the reference itself -------------------------------------------------------

def test_reference_agrees_with_torch():
    """torch.optim.AdamW in 64 bits takes the same steps."""
    gen = torch.Generator().manual_seed(1)
    p = torch.randn(500, generator=gen, dtype=torch.float64)
    q = p.clone().requires_grad_()
    opt = torch.optim.AdamW([q], lr=3e-3, betas=(0.9, 0.95), eps=1e-6, weight_decay=0.2)
    x, m, v = p.numpy(), np.zeros(500), np.zeros(500)
    for t in range(1, 6):
        g = torch.randn(500, generator=gen)
        q.grad = g.double()
        opt.step()
        x, m, v, _, _ = ref.step64(x, g.numpy(), m, v, t, 3e-3, (0.9, 0.95), 1e-6, 0.2, 1.0)
        assert np.allclose(x, q.detach().numpy(), rtol=1e-12, atol=1e-14)


def test_reference_words_are_uniform():
    """Means and neighbours' correlations of the random numbers, of elements and of steps."""
    n = 1 << 18
    e = np.arange(n)
    draws = []
    for t in (1, 2, 1000):
        w, y = ref.words(5, t, 3, e)
        draws += [(w >> np.uint32(12)) / 2.0 ** 20, (ref.turned(w) >> np.uint32(12)) / 2.0 ** 20, (y >> np.uint32(16)) / 2.0 ** 16]
    steps = np.array([ref.words(5, t, 0, np.array([77]))[0][0] >> np.uint32(12) for t in range(1, 4001)]) / 2.0 ** 20
    for u in draws + [steps]:
        assert abs(u.mean() - 0.5) < 6 / np.sqrt(12 * len(u)) + 2.0 ** -16
        for lag in (1, 8, 256):
            assert abs(np.corrcoef(u[:-lag], u[lag:])[0, 1]) < 6 / np.sqrt(len(u))
    for i, a in enumerate(draws):
        for b in draws[i + 1:]:
            assert abs(np.corrcoef(a, b)[0, 1]) < 6 / np.sqrt(n)
    hi = ref.words(5, 1, 3, e[:4096] + (1 << 32))[0]
    assert (hi != ref.words(5, 1, 3, e[:4096])[0]).mean() > 0.99


def test_reference_codes():
    """Values are e4m3's, right on average, exact where they have a code, never zero for v."""
    rng = np.random.default_rng(2)
    x = (rng.standard_normal(5000) * np.exp(3 * rng.standard_normal(5000))).astype(np.float32)
    total, rounds = np.zeros(5000), 400
    for t in range(rounds):
        y, s = ref.held(x, ref.words(1, t, 0, np.arange(5000))[0], False)
        total += y * np.repeat(s, 256)[:5000]
        assert (torch.from_numpy(y).float().to(torch.float8_e4m3fn).double().numpy() == y).all()
        assert np.abs(y).max() <= 256
    q = np.repeat(s, 256)[:5000] * 2.0 ** -9
    step = np.maximum(2.0 ** -3 * np.abs(x), q)
    assert (np.abs(total / rounds - x) < 6 * 0.5 * step / np.sqrt(rounds) + 2.0 ** -20 * step).all()
    again, _ = ref.held((y * np.repeat(s, 256)[:5000]).astype(np.float32), ref.words(9, 9, 9, np.arange(5000))[0], False,
                        ref.exponents(x))  # at the same scales
    assert (again == y).all()
    v, _ = ref.held(np.abs(x), ref.words(1, 1, 0, np.arange(5000))[0], True)
    assert v.min() >= 2.0 ** -9
    bad = x.copy()
    bad[7], bad[300] = np.inf, np.nan
    y, s = ref.held(bad, ref.words(1, 1, 0, np.arange(5000))[0], False)
    assert np.isnan(y[[7, 300]]).all() and np.isfinite(np.delete(y, [7, 300])).all()
