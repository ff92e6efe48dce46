"""The two launches of tg_reserve_device at the sizes and refusals that only they meet."""
import numpy as np
import pytest

from gpu_helpers import say
from paper_2606_06302_amd import tangram as tg
from test_tables_gpu import Admission, _gpu

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("what", ["pages", "capacity", "none", "exact"])
@pytest.mark.parametrize("B,L,H,Hp", [(70, 40, 4, 2), (9, 300, 2, 1), (3, 5, 256, 1)])
def test_too_few_pages(what, B, L, H, Hp):
    """More than 1024 tables: what is needed is exact, the tables are empty and no page id is written."""
    _gpu()
    ctx = np.arange(1, B + 1) * 29
    full = Admission(B, L, H, Hp, 16, ctx, seed=B)
    assert B * L * full.G > 1024
    kw = {"pages": dict(num_free=full.need - 1), "capacity": dict(capacity=full.need - 1),
          "none": dict(num_free=0, capacity=0), "exact": dict(num_free=full.need, capacity=full.need)}[what]
    a = Admission(B, L, H, Hp, 16, ctx, seed=B, **kw)
    got = a.run()
    if what == "exact":
        a.check_ok(got)
        return
    a.check_refused(got, tg.TG_ERR_BUFFER_TOO_SMALL if what == "capacity" else tg.TG_ERR_OUT_OF_PAGES)
    assert got["needed"][0] == full.need and np.all(got["pages"] == -77)


@pytest.mark.parametrize("B,L,H,Hp", [(2, 3, 256, 1), (3, 2, 256, 16), (40, 64, 8, 8), (5, 400, 129, 3), (600, 33, 2, 1)])
def test_wide_layers_and_many_workgroups(B, L, H, Hp):
    """One row per workgroup (more than 128 heads, up to the 256 that are taken), and more workgroups than one of them has
    threads for their sums."""
    _gpu()
    a = Admission(B, L, H, Hp, 16, 1 + np.arange(B) * 13 % 900, headroom=np.arange(B) % 40, seed=L, capacity=None)
    b = Admission(B, L, H, Hp, 16, a.ctx, headroom=a.headroom, seed=L, num_free=max(a.need, 13000))   # past the one-workgroup launch
    for x in (a, b):
        x.check_ok(x.run())
    say(f"{B * L} rows of {H} heads: {a.need} pages")


@pytest.mark.parametrize("bad", ["first", "last"])
def test_a_bad_value_in_the_first_and_the_last_workgroup(bad):
    _gpu()
    B, L = 600, 33
    a = Admission(B, L, 2, 1, 16, np.full(B, 50), seed=3)
    a.ratio[(0, 0, 0) if bad == "first" else (B - 1, L - 1, 1)] = np.nan
    got = a.run()
    a.check_refused(got, tg.TG_ERR_INVALID_ARG)
    assert np.all(got["pages"] == -77)
