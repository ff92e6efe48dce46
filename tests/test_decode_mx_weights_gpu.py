"""Weights of the attention over a quantised cache where the values cancel: a weight rounded to the result's type would be
most of such a result."""
import numpy as np
import pytest
import torch

from gpu_helpers import say

pytestmark = pytest.mark.gpu

if torch.cuda.is_available():
    from mx_helpers import Cache, attend, f64


@pytest.fixture(autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


@pytest.mark.parametrize("d,bits", [(128, (4, 4)), (128, (8, 8)), (64, (4, 8)), (64, (8, 4))])
@pytest.mark.parametrize("bins", [1, 3])
def test_bf16_weights_keep_more_bits_than_the_result(d, bits, bins):
    """Values 1 and -1 in turn, scores 0 and -delta: the result is tanh(delta / 2), the difference of two weights near 1.
    Off by: the scores' fp32 sums, (d + 1) 2^-23 of delta, twice in a weight; 2^-21 for the exponential; n 2^-23 for the
    sums; 2^-16 for a weight held in two bf16 parts, the first cut (2^-7 of it are left) and the second rounded (2^-9 of
    those); and half a step of the result, 2^-8 of it."""
    c = Cache([2, 3, 24, 40, 150], H=1, gqa=16, d=d, Hp=1, bits=bits, seed=d)
    one = np.zeros(d)
    one[0] = 1.0
    for b in range(c.B):
        for e in range(int(c.kv_len[b, 0, 0])):
            c.store(b, 0, 0, e, one * (e % 2), np.full(d, 1.0 - 2.0 * (e % 2)))
    c.pool.copy_(torch.from_numpy(c.host))
    delta = 2.0 ** -10 * 1.37 ** np.arange(16)
    q = torch.zeros(c.B, 16, d, dtype=torch.bfloat16, device="cuda")
    q[:, :, 0] = torch.from_numpy(-delta).to(q)
    out, lse, _ = c.decode(q, "bf16", bins=bins, sm_scale=1.0)
    o, qh, worst = f64(out), f64(q), 0.0
    for b in range(c.B):
        n = int(c.kv_len[b, 0, 0])
        k, v = c.rows(b, 0, 0, n)
        for j in range(16):
            want, _, size, qk = attend(qh[b, j], k, v, 1.0, 0.0)
            weight = 2 * qk * (d + 1) * 2.0 ** -23 + 2.0 ** -21 + n * 2.0 ** -23 + 2.0 ** -16
            bound = size * weight * 1.01 + np.abs(want) * 2.0 ** -8
            off = np.abs(o[b, j] - want)
            worst = max(worst, float((off / bound).max()))
            assert np.all(off <= bound), f"n {n} delta {delta[j]:.5f}: off {off.max():.2e}, bound {bound.max():.2e}"
    say(f"d {d} {bits} bins {bins}: {worst:.2f} of the bound")
