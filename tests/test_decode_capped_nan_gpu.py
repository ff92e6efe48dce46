"""NaN scores under a cap in the decode."""
import pytest
import torch

from test_score_mod_gpu import _gpu
from workloads import Geometry, custom

pytestmark = pytest.mark.gpu

if torch.cuda.is_available():
    from paper_2606_06302_amd import tangram as tg
    from paper_2606_06302_amd.runner import DecodeSession


@pytest.mark.parametrize("dtype,d,gqa", [("f32", 64, 2), ("f32", 64, 8), ("bf16", 128, 4), ("f32", 128, 8), ("bf16", 64, 8),
                                         ("bf16", 64, 1), ("bf16", 64, 4), ("f32", 128, 1)])
@pytest.mark.parametrize("fused", [False, True])
def test_a_nan_score_makes_its_heads_nan_and_no_other(dtype, d, gqa, fused):
    """A NaN key is in the scores of its KV head's query heads, a NaN query in its own: those outputs and log-sums are NaN,
    all others as without, bit for bit."""
    _gpu()
    import numpy as np
    wl = custom(57, Geometry(1, 2, 2 * gqa, d, 16, 1), 2, dtype, 200, ratio=np.ones((2, 1, 2)), q_scale=1.0)
    s = DecodeSession(wl, mode=tg.TG_PLAN_AOT_FILL, n_bins=8, fill="host", softcap=4.0, fused_merge=fused)

    def run():
        s.run_step()
        torch.cuda.synchronize()
        return s.out[0].clone(), s.lse[0].clone()
    out, lse = run()
    page = int(s.t.pt_pages[int(s.t.pt_offsets[int(s.t.group_of[0, 0])])])       # request 0, KV head 0
    keep = s.pool[page, 0, 0, 5, 7].clone()
    s.pool[page, 0, 0, 5, 7] = float("nan")
    got, glse = run()
    assert bool(torch.isnan(got[0, :gqa]).all()) and bool(torch.isnan(glse[0, :gqa]).all())
    assert torch.equal(got[0, gqa:], out[0, gqa:]) and torch.equal(glse[0, gqa:], lse[0, gqa:])
    assert torch.equal(got[1], out[1]) and torch.equal(glse[1], lse[1])
    s.pool[page, 0, 0, 5, 7] = keep
    s.q[0, 1, gqa, 3] = float("nan")
    got, glse = run()
    assert bool(torch.isnan(got[1, gqa]).all()) and bool(torch.isnan(glse[1, gqa]))
    got[1, gqa], glse[1, gqa] = out[1, gqa], lse[1, gqa]
    assert torch.equal(got, out) and torch.equal(glse, lse)
