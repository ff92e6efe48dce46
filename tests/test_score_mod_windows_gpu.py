"""Windows inside the chunk, as the header writes them: with and without the history."""
import numpy as np
import pytest
import torch

from test_score_mod_gpu import Prefill, _gpu, cuda

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("split", [False, True])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("window", [1, 5, 64, 70, 1000])
@pytest.mark.parametrize("clamped", [True, False])
def test_windows(clamped, window, d, split):
    """key_begin = max(i + 1 - window, 0): no row sees the history.  Without the max: rows before the window-th see all of it."""
    _gpu()
    C = 150
    p = Prefill(51, 2, 3, d, 2, 2, C, (40, 500), "causal", 8.0 if window == 64 else 0.0, tokens=[C, 101], split=split)
    begin = np.tile(np.arange(C) + 1 - window, (2, 1))
    if clamped:
        begin = np.maximum(begin, 0)
    p.begin, p.keep[1] = begin, cuda(begin)
    p.s.mod.key_begin = p.keep[1].data_ptr()
    p.s.run()
    torch.cuda.synchronize()
    p.check(f"window {window} clamped {clamped} d{d} split {split}")
    chunk, hist, _ = p.seen(0)
    assert chunk.sum(1).max() == min(window, C) and hist.sum() == (0 if clamped else min(window - 1, C))
