"""Values at the ends of what the AdamW step's arguments allow (GPU)."""
import numpy as np
import pytest
import torch

import adamw_reference as ref
from paper_2412_07210_amd import AdamW, AdamWConfig
from test_gpu_adamw import DEV, randn

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
