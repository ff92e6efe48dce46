"""Bins of a plan over a quantised cache, on both sides of every border of the rule (needs a device for its CUs and the
kernels' occupancy; nothing is launched)."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

if torch.cuda.is_available():
    from mx_helpers import DTYPE, TG, Cache, fmt
    from paper_2606_06302_amd import tangram as tg


@pytest.fixture(autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def lengths(pages, heads=4, layers=2, seed=0):
    """[1][layers][heads] lengths of `pages` pages in layer 1, odd ones among them; the other layer's do not count."""
    rng = np.random.default_rng(seed)
    share = np.full(heads, pages // heads)
    share[:pages % heads] += 1
    kv = np.full((1, layers, heads), 77, np.int32)
    kv[0, 1] = np.maximum(1, share * 16 - rng.integers(0, 16, heads))
    return kv


@pytest.mark.parametrize("dtype,d,gqa,bits,most", [("bf16", 128, 4, (4, 4), 3), ("bf16", 128, 4, (8, 8), 3), ("bf16", 64, 8, (8, 4), 3),
                                                   ("f32", 64, 2, (4, 4), 3), ("bf16", 128, 16, (8, 4), 2), ("f32", 128, 5, (8, 4), 2)])
def test_bins_around_the_borders(dtype, d, gqa, bits, most):
    """Three pages a bin at least, two workgroups a CU, three from 80 pages a bin on where `most` fit a CU."""
    cus = torch.cuda.get_device_properties(0).multi_processor_count
    g = tg.tg_geometry(2, 4, 4 * gqa, d, 16, 2)
    bins = lambda pages: tg.tg_decode_mx_bins(g, TG[dtype], fmt(bits), 0, 1, 1, lengths(pages, seed=pages))
    assert tg.tg_decode_mx_bins(g, TG[dtype], fmt(bits)) == 2 * cus
    for pages, want in ((4, 2), (5, 2), (6, 2), (7, 3), (6 * cus - 3, 2 * cus - 1), (6 * cus - 2, 2 * cus), (6 * cus, 2 * cus),
                        (6 * cus + 1, 2 * cus), (240 * cus - 1, 2 * cus), (240 * cus, most * cus), (1000 * cus, most * cus)):
        assert bins(pages) == want, pages
    one = tg.tg_geometry(1, 1, gqa, d, 16, 1)
    assert tg.tg_decode_mx_bins(one, TG[dtype], fmt(bits), 0, 1, 0, np.ones((1, 1, 1), np.int32)) == 1
    # lengths whose sum is past 32 bits
    assert tg.tg_decode_mx_bins(g, TG[dtype], fmt(bits), 0, 3, 1, np.full((3, 2, 4), 2 ** 31 - 1, np.int32)) == most * cus


@pytest.mark.parametrize("dtype,d,gqa,bits", [("bf16", 128, 1, (8, 4)), ("bf16", 128, 2, (8, 4)), ("bf16", 128, 11, (4, 4)),
                                              ("bf16", 128, 12, (4, 4)), ("bf16", 128, 12, (8, 8)), ("f32", 64, 16, (8, 8))])
def test_the_workgroups_of_many_bins_run_together(dtype, d, gqa, bits):
    """The last workgroup starts before the first ends: as many fit a CU as the rule says, also where it is a close fit in
    LDS."""
    c = Cache([1 << 14] * 16, H=8, gqa=gqa, d=d, Hp=8, bits=bits, headroom=0, fill=False)
    c.kv_len[:] = 1 << 13                                  # what is attended to does not matter here, only how long
    cus = torch.cuda.get_device_properties(0).multi_processor_count
    assert int((c.kv_len // 16).sum()) >= 240 * cus
    bins = tg.tg_decode_mx_bins(c.geom, TG[dtype], c.fmt, 0, c.B, 0, c.kv_len)
    assert bins in (2 * cus, 3 * cus)
    # every head's table holds its pages: the longest head of the one group reserved for all
    assert np.all(np.diff(c.offsets) >= (1 << 13) // 16)
    q = torch.zeros(c.B, 8 * gqa, d, dtype=DTYPE[dtype], device="cuda")
    ts = torch.zeros(2 * bins, dtype=torch.int64, device="cuda")
    for _ in range(3):                                     # the first call loads the code
        c.decode(q, dtype, bins=bins, timestamps=ts)
    start, end = ts.view(-1, 2).cpu().numpy().T
    assert start.max() < end.min(), f"{bins} bins: the last starts {(start.max() - end.min()) / 100} us after the first ends"
