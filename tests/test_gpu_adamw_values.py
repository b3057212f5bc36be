"""Values at the ends of what the AdamW step's arguments allow (GPU)."""
import numpy as np
import pytest
import torch

import adamw_reference as ref
from paper_2412_07210_amd import AdamW, AdamWConfig
from test_gpu_adamw import DEV, Run, randn

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n", [300, 5000])
def test_pack_takes_v_by_its_size(n):
    """-0, which is >= 0, and negative values beside a large one of their block: held at
    the smallest code above zero at least, as positive ones are, so that the next step's
    root is one of a positive number.  m keeps its signs."""
    m, v = randn(n, 31), randn(n, 32).exp_()
    v[::3] *= -1e-12
    v[1::3] *= 1e-12
    v[::5] = -0.0
    v[7], v[11], v[200] = -1e4, 1e4, -float("nan")
    m[::2] = -0.0
    m = [torch.cat([m, m.new_zeros(4)])[:n]]
    opt = AdamW(AdamWConfig([n], "f32", state="e4m3", betas=(0.9, 0.95)), DEV)
    state = opt.pack(m, [v], seed=5)
    back = opt.unpack(state)[1][0].cpu().double().numpy()
    w, _ = ref.words(5, 0, 0, np.arange(n))
    for x, codes, scale, second in ((m[0], state.exp_avg[0], state.exp_avg_scale[0], False),
                                    (v.abs(), state.exp_avg_sq[0], state.exp_avg_sq_scale[0], True)):
        value, s = ref.held(x.cpu().numpy(), w, second)
        assert (scale.cpu().double().numpy() == s).all()
        assert np.array_equal(codes.float().cpu().double().numpy(), value, equal_nan=True)
    fine = np.arange(n) != 200
    assert np.isnan(back[200]) and (back[fine] >= np.repeat(s, 256)[:n][fine] * 2.0 ** -9).all()
    p = [torch.zeros(n, device=DEV)]
    opt.step(p, [torch.zeros(n, device=DEV)], state, 1e-3)
    assert torch.isfinite(p[0].cpu()[torch.from_numpy(fine)]).all()
    opt.close()


@pytest.mark.parametrize("missing", [(), (1,)], ids=["fused", "apart"])
@pytest.mark.parametrize("state", ["f32", "e4m3"])
@pytest.mark.parametrize("factor,decay", [(1e39, 0.0), (1e300, 0.0), (1e40, 1e-41), (1e-46, 1e45), (2.5, 0.1)])
def test_decay_factors_of_any_size(state, factor, decay, missing):
    """lambda d_k is taken in 64 bits: factors beyond fp32's range are factors."""
    run = Run([700, 300, 5000], "f32", None, state, seed=33, no_grad=missing, weight_decay=decay, decay=[factor] * 3)
    old, g = run.params[0].double().cpu().numpy(), run.grads[0].cpu().numpy()
    run.opt.step(run.params, run.grads, run.state, 1e-2)
    p, _, _, step, _ = ref.step64(old, g, np.zeros(700), np.zeros(700), 1, 1e-2, (0.9, 0.95), 1e-8, decay * factor, 1.0)
    assert np.isfinite(p).all()
    ref.assert_params(run.params[0], p, step, f"{factor} {decay}")
    run.close()


@pytest.mark.parametrize("std", [1e-21, 1e-19, 1e-18, 1e-17])
@pytest.mark.parametrize("beta2", [0.95, 0.999, 0.9999, 0.999999])
@pytest.mark.parametrize("state", ["f32", "e4m3"])
def test_steps_where_the_roots_argument_is_subnormal(state, beta2, std):
    """With the smallest eps and few steps taken, sqrt(v / (1 - beta2^t)) of a v below
    2^-126 shows beside eps.  Parameters of zero: the step is all that is compared."""
    run = Run([3000, 257], "f32", None, state, seed=34, std=std, eps=1e-12, betas=(0.9, beta2))
    for t in range(3):
        run.draw(t)
        run.flat_p.zero_()
        run.step(lr=1e4)
    run.close()
