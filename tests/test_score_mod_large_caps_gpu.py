"""tg_prefill_mod where scores come near a large cap: the weight of a key goes by its score alone, whatever else its block
of keys holds, and its exponent is as exact as fp32 has it.

Scores are made of two products, so that their own error is counted: x = sm_scale * q . k with both products exact in
fp32, their sum rounded once (2^-24 x).  The exponent's error, in units of |z| <= |x|: the score's rounding, the scale
over the cap and its product, the cap in log2 units and its product and difference (6 of 2^-24, 3.6e-7) and tanh's 2e-7,
or a polynomial's 2^-13 in all: e = max(2^-13, 2e-7 |x|) + 3.6e-7 |x|.  (The row's reference is off by as much for all its
keys alike, which cancels.)  The probabilities are rounded to bf16 (2^-8) for the numerator and not for the sum: with
W = sum_k p_k |v_k| / sum_k p_k,
  |out - o| <= 2^-8 |o| + 2^-8 W + e (W + |o|) + 1e-5 W (the exponentials and fp32 sums)."""
import math

import numpy as np
import pytest
import torch

from gpu_helpers import say
from test_score_mod_gpu import Prefill, _gpu, attend, f64

pytestmark = pytest.mark.gpu


def one_head(cap, d, split, C=128):
    """Every row sees all of its chunk's C keys, no history, cap over the scores."""
    return Prefill(31, 1, 2, d, 1, 1, C, 50, "bidirectional", cap, hist=0, split=split)


@pytest.mark.parametrize("split", [False, True])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("cap", [50.0, 1e3, 1e4, 1e5, 1e6])
def test_equal_scores_have_equal_weights(cap, d, split):
    """Keys of one score in blocks of 32 that differ in what else they hold: nothing, or a score of -0.55 of the cap."""
    _gpu()
    p = one_head(cap, d, split)
    s = p.s
    s.q.zero_(), s.k_new.zero_(), s.v_new.fill_(1.0)
    unit = 2.0 ** math.floor(math.log2(cap / 100))               # x = unit * k0
    s.q[..., 0] = unit * (8 if d == 64 else 8 * math.sqrt(2))    # sm_scale = 1 / 8, or 1 / 8 sqrt 2: a rounding of q is every key's
    for part in (0.3, 0.5, 0.63):
        s.k_new[0, :, 0, 0] = round(part * cap / unit)
        for b in (1, 2):
            s.k_new[0, 32 * b + 5, 0, 0] = -round(0.55 * cap / unit)
            s.v_new[0, 32 * b:32 * b + 32] = -1.0
        p.s.run()
        torch.cuda.synchronize()
        # 64 keys of value 1, 62 of value -1, two of no weight: the probabilities are 1 before they are rounded to bf16
        o, gap = 2 / 126, cap * (math.tanh(part) + math.tanh(0.55))
        got = f64(s.out)
        assert gap > 30                                          # e^-30 of the two
        # equal scores, equal bits: what is left is the division and the result's rounding
        assert np.all(np.abs(got - o) <= 2.0 ** -8 * o + 1e-6), (part, got.min(), got.max(), o)


@pytest.mark.parametrize("split", [False, True])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("cap", [50.0, 60.0, 80.0, 1e3, 1e4])
@pytest.mark.parametrize("part", [0.2, 0.33, 0.45, 0.6, 0.7, 0.9])
def test_scores_a_fifth_to_three_fifths_of_the_cap(part, cap, d, split):
    """Scores a few units apart around `part` of the cap; every other block also holds one far below."""
    _gpu()
    p = one_head(cap, d, split)
    s, rng = p.s, np.random.default_rng(int(100 * part))
    unit = 2.0 ** math.floor(math.log2(cap / 100))
    s.q.zero_(), s.k_new.zero_()
    s.q[..., 0], s.q[..., 1] = 8 * unit, 8.0
    k = np.zeros((128, d))
    k[:, 0] = round(part * cap / unit)
    k[:, 1] = rng.normal(size=128) * 2
    k[37, 0] = k[101, 0] = -round(0.55 * cap / unit)
    s.k_new[0, :, 0] = torch.from_numpy(k).bfloat16().cuda()
    sign = np.where((np.arange(128) // 32) % 2 == 0, 1.0, -1.0)
    s.v_new[0, :, 0] = torch.from_numpy(sign[:, None] * (1 + rng.random((128, d)))).bfloat16().cuda()
    p.s.run()
    torch.cuda.synchronize()
    scale = 1 / math.sqrt(d)
    k, v, got = f64(s.k_new)[0, :, 0], f64(s.v_new)[0, :, 0], f64(s.out)
    x = f64(s.q)[0, 0, :1] @ k.T * scale
    x = np.abs(x).max()
    e = max(2.0 ** -13, 2e-7 * x) + 3.6e-7 * x
    o, w = attend(f64(s.q)[0, 0, :1], k, v, np.ones((1, 128), bool), scale, cap)
    tol = 2.0 ** -8 * np.abs(o) + (2.0 ** -8 + 1e-5) * w + e * (w + np.abs(o))
    err = np.abs(got[0] - o[0])
    assert np.all(err <= tol[0]), (float((err / tol[0]).max()), e)
    say(f"cap {cap} part {part} d{d} split {split}: {float((err / tol[0]).max()):.2f} of the tolerance")
