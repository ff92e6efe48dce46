"""The byte counts of sessions over a quantised cache (CPU only: nothing is launched)."""
import numpy as np
import pytest
import torch

from oracle import mx
from paper_2606_06302_amd import tangram as tg
from paper_2606_06302_amd.runner import CompressSession, PrefillSession, Tables
from workloads import Geometry, custom


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("bits", [(4, 4), (8, 4), (8, 8)])
def test_bytes_of_what_is_stored(d, dtype, bits):
    g = Geometry(2, 4, 8, d, 16, 2)
    wl = custom(5, g, 2, "bf16" if dtype == "bf16" else "f32", (30, 60), chunk_len=8)
    t = Tables(wl, device="cpu")
    form = {4: tg.TG_MX_FP4, 8: tg.TG_MX_FP8}
    fmt = tg.make_mx_format(form[bits[0]], form[bits[1]])
    entry, esz = mx.slab_bytes(d, *bits) // 16, 4 if dtype == "f32" else 2
    kv = t.kv_len.astype(np.int64)
    assert t.kv_bytes() == int(kv.sum()) * 2 * d * esz and t.kv_bytes(1) == int(kv[:, 1].sum()) * 2 * d * esz
    assert t.kv_bytes(mx=fmt) == int(kv.sum()) * entry and t.kv_bytes(0, fmt) == int(kv[:, 0].sum()) * entry
    pool = torch.zeros(t.pool_pages * tg.tg_mx_page_bytes(g, fmt), dtype=torch.uint8)
    tokens = np.full(2, 8, np.int32)
    c = CompressSession(wl, t, pool, wl.ctx_len - tokens, tokens, device="cpu", mx=fmt)
    kept = int(c.plan["keep_count"].sum())
    assert c.traffic_bytes() == kept * (2 * d * esz + entry + 8) + 16 * 4 * 4
    if dtype == "bf16":
        rows, coded = (PrefillSession(wl, tables=t, device="cpu", fill="host", **kw) for kw in ({}, dict(mx=fmt, mx_pool=pool)))
        chunk = 2 * d * 2 * 2 * 8 * (8 + 4)
        assert rows.min_hbm_bytes() == chunk + int(kv[:, 0].sum()) * 2 * d * 2
        assert coded.min_hbm_bytes() == chunk + int(kv[:, 0].sum()) * entry
