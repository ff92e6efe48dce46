"""What a row of tg_prefill_mod does not see does not reach its output, bit for bit, also where the scores are capped: the
way a cap is computed goes by the row's own scores."""
import numpy as np
import pytest
import torch

from gpu_helpers import say
from test_score_mod_gpu import Prefill, _gpu, cuda

pytestmark = pytest.mark.gpu

# caps over scores of about 1.4 standard deviations: most rows within a third of the cap, some beyond it, and all far beyond
CAPS = [50.0, 6.0, 0.5]
BAD = [300.0, -3e4, float("inf"), -float("inf"), float("nan")]


def runs(p):
    p.s.out.fill_(float("nan"))
    p.s.run()
    torch.cuda.synchronize()
    return p.s.out.clone()


def same(a, b):
    return torch.equal(a.nan_to_num(1e9), b.nan_to_num(1e9))


@pytest.mark.parametrize("split", [False, True])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("cap", CAPS)
def test_another_documents_keys_and_values(cap, d, split):
    """Tokens 50.. see neither the history nor tokens 0..49, which share their key tiles (and, with four query heads
    per KV head, row 49's wave)."""
    _gpu()
    p = Prefill(21, 2, 4, d, 2, 1, 96, 200, "causal", cap, q_scale=2.0, split=split)
    begin = np.full((1, 96), -1)
    begin[0, 50:] = 50
    p.keep[1] = cuda(begin)
    p.s.mod.key_begin, p.begin = p.keep[1].data_ptr(), begin
    clean = runs(p)
    p.check("finite")
    k, v, pool = p.s.k_new.clone(), p.s.v_new.clone(), p.s.pool.clone()
    ids = torch.from_numpy(p.t.pt_pages.astype(np.int64)).cuda()
    for bad in BAD:
        p.s.k_new[0, 10:50] = bad
        assert torch.equal(runs(p)[0, 50:], clean[0, 50:]), ("keys", bad)
        p.s.v_new[0, 20:50] = bad
        assert torch.equal(runs(p)[0, 50:], clean[0, 50:]), ("values", bad)
        p.s.pool[ids] = bad
        assert torch.equal(runs(p)[0, 50:], clean[0, 50:]), ("history", bad)
        p.s.k_new.copy_(k), p.s.v_new.copy_(v), p.s.pool.copy_(pool)
    # values alone: nothing but the outputs that see them
    p.s.v_new[0, 49, 0, 3] = float("inf")
    got = runs(p)
    got[0, 49, :4, 3] = clean[0, 49, :4, 3]
    assert torch.equal(got, clean)
    say(f"documents cap {cap} d{d} split {split}")


@pytest.mark.parametrize("split", [False, True])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("cap", CAPS)
def test_the_rest_of_the_last_page_and_of_the_chunk(cap, d, split):
    """Rows of the last history page past the retained ones, and tokens past the request's, hold anything."""
    _gpu()
    p = Prefill(22, 2, 4, d, 2, 2, 70, (100, 300), "causal", cap, q_scale=2.0, tokens=[70, 33], split=split, nan=False)
    finite = torch.isfinite(p.s.pool)                # the rest of the pages is NaN
    p.s.pool[~finite] = 0
    clean = runs(p)
    p.pool = p.s.pool.double().cpu().numpy()
    p.check("zeros")
    for bad in BAD:
        p.s.pool[~finite] = bad
        for x in (p.s.k_new, p.s.v_new):
            x[1, 33:] = bad
        assert same(runs(p), clean), bad


@pytest.mark.parametrize("split", [False, True])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("cap", CAPS)
def test_other_rows_of_the_wave(cap, d, split):
    """A row's output goes by its own query: others' queries, far greater or infinite, change nothing."""
    _gpu()
    p = Prefill(23, 1, 4, d, 1, 1, 40, 150, "any", cap, q_scale=2.0, split=split)
    clean = runs(p)
    q = p.s.q.clone()
    odd = torch.arange(40, device="cuda") % 2 == 1
    for scale in (40.0, 3000.0, float("inf")):
        p.s.q[:, odd] = q[:, odd] * scale
        got = runs(p)
        assert torch.equal(got[:, ~odd], clean[:, ~odd]), scale
        p.s.q.copy_(q)
    # one head's queries
    p.s.q[:, :, 1] = q[:, :, 1] * 100
    got = runs(p)
    rest = [0, 2, 3]
    assert torch.equal(got[:, :, rest], clean[:, :, rest])


@pytest.mark.parametrize("split", [False, True])
@pytest.mark.parametrize("d", [64, 128])
def test_history_of_some_rows_under_a_cap(d, split):
    _gpu()
    for cap in CAPS:
        p = Prefill(24, 1, 4, d, 1, 1, 40, 100, "causal", cap, q_scale=2.0, split=split)
        begin = np.where(np.arange(40) % 2 == 0, -1, 0)[None]
        p.keep[1] = cuda(begin)
        p.s.mod.key_begin = p.keep[1].data_ptr()
        clean = runs(p)
        page = int(p.t.pt_pages[int(p.t.pt_offsets[1])])
        p.s.pool[page, 1, 0, 3, 5] = float("inf")
        got = runs(p)
        assert bool(torch.isinf(got[0, 0::2, :, 5]).all())
        got[0, 0::2, :, 5] = clean[0, 0::2, :, 5]
        assert torch.equal(got, clean)
        p.s.pool[page, 0, 0, 3] = float("nan")
        assert torch.equal(runs(p)[0, 1::2], clean[0, 1::2])
