"""The cap itself: a request of one token has its capped score as the log-sum of every query head."""
import numpy as np
import pytest
import torch

from gpu_helpers import say
from test_score_mod_gpu import _gpu
from workloads import Geometry, custom

pytestmark = pytest.mark.gpu

if torch.cuda.is_available():
    from paper_2606_06302_amd import tangram as tg
    from paper_2606_06302_amd.runner import DecodeSession


@pytest.mark.parametrize("cap", [1e-3, 1.0, 30.0, 50.0, 1e4, 1e6])
@pytest.mark.parametrize("gqa", [1, 8])
def test_capped_scores(cap, gqa):
    """fp32, head_dim 64: s = q . k / 8 is exact.  In units of the value: the cap's reciprocal scale and its product (2 of
    2^-24), tanh 2e-7, the cap in log2 units and its product (2), log2 units to natural ones (2): 5.6e-7, one more for the
    sum with log 1 = 0."""
    _gpu()
    B, H = 64, 8
    wl = custom(81, Geometry(1, H, H * gqa, 64, 16, 2), B, "f32", 1)
    s = DecodeSession(wl, mode=tg.TG_PLAN_AOT_FILL, n_bins=64, fill="host", softcap=cap)
    rng = np.random.default_rng(int(gqa))
    worst = 0.0
    s.pool.zero_()
    s.pool[:, 0, :, :, 0] = 1.0
    for _ in range(40):
        # from far below the cap to far past it, half of them where the two forms of tanh meet
        x = cap * np.concatenate([np.exp(rng.uniform(-12, 3, 32 * H * gqa)), rng.uniform(0.5, 0.8, 32 * H * gqa)])
        x *= rng.choice([-1.0, 1.0], x.size)
        q = torch.zeros(1, B, H * gqa, 64)
        q[0, :, :, 0] = torch.from_numpy(x.reshape(B, H * gqa) * 8).float()
        s.q.copy_(q)
        s.run_step()
        torch.cuda.synchronize()
        want = cap * np.tanh(q[0, :, :, 0].double().numpy() / 8 / cap)
        got = s.lse[0].double().cpu().numpy()
        worst = max(worst, float((np.abs(got - want) / np.abs(want)).max()))
    say(f"cap {cap} gqa {gqa}: {worst:.2e}")
    assert worst <= 6.2e-7
