"""Decode attention over a quantised cache against 64 bits, on the values that the cache stands for."""
import math

import numpy as np
import pytest
import torch

from gpu_helpers import say

pytestmark = pytest.mark.gpu

if torch.cuda.is_available():
    from mx_helpers import DTYPE, FORMATS, TG, Cache, check_decode, f64
    from paper_2606_06302_amd import tangram as tg
    from paper_2606_06302_amd.device import to_device
else:
    FORMATS = [(4, 4), (8, 4), (4, 8), (8, 8)]


@pytest.fixture(autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def queries(c, dtype, scale=1.0, seed=1):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(c.B, c.H * c.gqa, c.d, generator=gen, device="cuda") * scale).to(DTYPE[dtype])


@pytest.mark.parametrize("bits", FORMATS)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("gqa", [1, 5, 16])
def test_decode(bits, dtype, d, gqa):
    """Lengths from one token on, around pages and steps, in a pool whose other bytes stand for NaN."""
    c = Cache([1, 2, 15, 16, 17, 31, 33, 70, 129, 300, 1000], H=4, gqa=gqa, d=d, Hp=2, bits=bits, L=2, seed=d + gqa)
    q = queries(c, dtype)
    out, lse, plan = c.decode(q, dtype, layer=1)
    worst = check_decode(c, q, out, lse, dtype, layer=1, what=f"{bits} {dtype} d {d} gqa {gqa}")
    say(f"{bits} {dtype} d {d} gqa {gqa}: {plan['num_partials']} partials, {worst:.2f} of the bound")


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("f32", 64), ("bf16", 64), ("f32", 128)])
@pytest.mark.parametrize("bins", [1, 7, 64, 1024])
def test_partitions_and_merges(dtype, d, bins):
    """Any number of bins; arrival counters change nothing."""
    c = Cache([40, 700, 2500, 3], H=2, gqa=3, d=d, Hp=1, bits=(8, 4), seed=bins)
    q = queries(c, dtype)
    out, lse, plan = c.decode(q, dtype, bins=bins)
    check_decode(c, q, out, lse, dtype, what=f"bins {bins}")
    out2, lse2, _ = c.decode(q, dtype, bins=bins, counters=True)
    assert torch.equal(out, out2) and torch.equal(lse, lse2)
    for mode in (tg.TG_PLAN_NAIVE, tg.TG_PLAN_AOT, tg.TG_PLAN_UNIFORM):
        out3, lse3, _ = c.decode(q, dtype, bins=bins, mode=mode, counters=True)
        check_decode(c, q, out3, lse3, dtype, what=f"bins {bins} mode {mode}")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("softcap,sm_scale,qs", [(0.0, 0.03, 5.0), (30.0, 0.0, 8.0), (1e-3, 0.0, 1.0), (50.0, 0.5, 20.0)])
def test_scales_and_caps(dtype, softcap, sm_scale, qs):
    c = Cache([9, 130, 800], H=2, gqa=4, d=128, Hp=2, bits=(4, 8), seed=5)
    q = queries(c, dtype, qs)
    out, lse, _ = c.decode(q, dtype, softcap=softcap, sm_scale=sm_scale)
    check_decode(c, q, out, lse, dtype, softcap=softcap, sm_scale=sm_scale, what=f"cap {softcap} scale {sm_scale}")


@pytest.mark.parametrize("bits", FORMATS)
@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("f32", 64), ("f32", 128), ("bf16", 64)])
def test_append_in_the_call(bits, dtype, d):
    """Several steps of one open-ended plan: the bytes, lengths and outputs of tg_append_mx followed by tg_decode_mx."""
    lens = [1, 14, 15, 16, 31, 32, 127, 128, 500]
    a, b = (Cache(lens, H=2, gqa=2, d=d, Hp=2, bits=bits, L=2, headroom=5, seed=11) for _ in range(2))
    la, lb = (to_device(a.kv_len, "cuda") for _ in range(2))
    gen = torch.Generator(device="cuda").manual_seed(2)
    for step in range(5):
        k, v = (torch.randn(a.B, a.H, d, generator=gen, device="cuda").to(DTYPE[dtype]) for _ in range(2))
        if step == 3:
            k[2, 1, 7], v[3, 0, 40] = float("nan"), float("inf")     # stored, and NaN wherever they are attended to
        q = queries(a, dtype, seed=step)
        tg.tg_append_mx(tg.make_append_args(a.geom, a.B, 1, TG[dtype], k, v, a.pool, *a.tables, la), a.fmt)
        out, lse, _ = a.decode(q, dtype, layer=1, open_end=True, live=la, counters=True)
        full = torch.zeros(1, dtype=torch.int32, device="cuda")
        out2, lse2, _ = b.decode(q, dtype, layer=1, open_end=True, live=lb, k_tok=k, v_tok=v, full=full)
        assert int(full) == 0 and torch.equal(la, lb) and torch.equal(a.pool, b.pool)
        assert np.array_equal(f64(out), f64(out2), equal_nan=True) and np.array_equal(f64(lse), f64(lse2), equal_nan=True)
        if step < 3:
            check_decode(a, q, out, lse, dtype, layer=1, lens=a.kv_len[:, 1] + step + 1, host=a.pool.cpu().numpy())
    bad = torch.isnan(out).any(-1)
    assert bool(bad[2, 2:4].all()) and bool(bad[3, 0:2].all()) and int(bad.sum()) == 4


def test_append_past_the_table():
    c = Cache([16, 40], H=2, gqa=2, d=64, Hp=1, headroom=1, seed=3)
    capacity = np.diff(c.offsets).reshape(2, 2)[:, c.group_of[0]] * 16
    n = c.kv_len.copy()
    n[0, 0] = capacity[0]
    for b, h in ((0, 0), (0, 1)):          # rows up to the capacity, not only the retained ones
        for e in range(int(c.kv_len[b, 0, h]), int(capacity[b, h])):
            c.store(b, 0, h, e, np.ones(64), np.ones(64) * e)
    c.pool.copy_(torch.from_numpy(c.host))
    live, full = to_device(n, "cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    k, v = (torch.randn(2, 2, 64, device="cuda").bfloat16() for _ in range(2))
    q = queries(c, "bf16")
    out, lse, _ = c.decode(q, "bf16", open_end=True, live=live, k_tok=k, v_tok=v, full=full)
    for h in range(2):
        c.store(1, 0, h, int(n[1, 0, h]), f64(k)[1, h], f64(v)[1, h])
    n[1] += 1
    assert int(full) == 1 and np.array_equal(live.cpu().numpy(), n) and np.array_equal(c.pool.cpu().numpy(), c.host)
    check_decode(c, q, out, lse, "bf16", lens=n[:, 0])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_scores_of_minus_infinity(dtype):
    """Scores that overflow to -inf have no weight, also where they fill whole steps and waves."""
    c = Cache([400], H=1, gqa=2, d=64, Hp=1, bits=(8, 8), seed=4)
    n = int(c.kv_len[0, 0, 0])
    for e in range(n):
        c.store(0, 0, 0, e, np.where(np.arange(64) < 2, -1.0 if e < n - 3 else 0.0, 0.5), np.full(64, float(e % 13)))
    c.pool.copy_(torch.from_numpy(c.host))
    q = torch.ones(1, 2, 64, device="cuda").to(DTYPE[dtype])
    q[0, 0, :2] = torch.finfo(q.dtype).max
    for bins in (1, 3):
        out, lse, _ = c.decode(q, dtype, bins=bins)
        v = c.rows(0, 0, 0, n)[1]
        assert np.allclose(f64(out)[0, 0], v[-3:].mean(0), rtol=2.0 ** -8)
        assert abs(float(lse[0, 0]) - (31 / 8 + math.log(3))) < 1e-5
    # no score above it: zeros, and the smallest lse, however the head is cut
    for e in range(n - 3, n):
        c.store(0, 0, 0, e, np.where(np.arange(64) < 2, -1.0, 0.5), np.ones(64))
    c.pool.copy_(torch.from_numpy(c.host))
    for bins in (1, 3, 20):
        for counters in (False, True):
            out, lse, _ = c.decode(q, dtype, bins=bins, counters=counters)
            assert bool((out[0, 0] == 0).all()) and float(lse[0, 0]) == -torch.finfo(torch.float32).max
            assert bool(torch.isfinite(out).all())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_infinite_scores_under_a_cap(dtype):
    c = Cache([100], H=1, gqa=1, d=64, Hp=1, bits=(8, 8), seed=6)
    n = int(c.kv_len[0, 0, 0])
    for e in range(n):
        sign = 1.0 if e % 2 else -1.0
        c.store(0, 0, 0, e, np.where(np.arange(64) == 0, sign, 0.25), np.full(64, sign))
    c.pool.copy_(torch.from_numpy(c.host))
    q = torch.ones(1, 1, 64, device="cuda").to(DTYPE[dtype])
    q[0, 0, 0] = float("inf")
    out, lse, _ = c.decode(q, dtype, softcap=2.0)
    up, down = (n // 2) * math.exp(2.0), (n - n // 2) * math.exp(-2.0)
    # a weight off by half a step (2^-8) either way, the result by another
    assert np.all(np.abs(f64(out) - (up - down) / (up + down)) <= 2.0 ** -7)
    assert abs(float(lse) - math.log(up + down)) < 1e-5


def test_timestamps_and_bins():
    c = Cache([900, 30], H=2, gqa=2, d=128, Hp=2, bits=(4, 4))
    most = tg.tg_decode_mx_bins(c.geom, tg.TG_BF16, c.fmt)
    some = tg.tg_decode_mx_bins(c.geom, tg.TG_BF16, c.fmt, 0, 2, 0, c.kv_len)
    assert 1 <= some < most and most % torch.cuda.get_device_properties(0).multi_processor_count == 0
    q = queries(c, "bf16")
    ts = torch.zeros(2 * 40, dtype=torch.int64, device="cuda")
    out, lse, plan = c.decode(q, "bf16", bins=40, timestamps=ts)
    check_decode(c, q, out, lse, "bf16")
    t = ts.view(-1, 2).cpu().numpy()
    assert np.all(t[:plan["num_bins"], 0] > 0) and np.all(t[:, 1] >= t[:, 0])


def test_captured_step():
    """A step (append and attention) captured once and replayed, on another stream, beside eager work."""
    c = Cache([60, 7, 400], H=2, gqa=4, d=128, Hp=2, bits=(8, 4), headroom=40, seed=8)
    e = Cache([60, 7, 400], H=2, gqa=4, d=128, Hp=2, bits=(8, 4), headroom=40, seed=8)
    lc, le = (to_device(c.kv_len, "cuda") for _ in range(2))
    k, v = (torch.randn(3, 2, 128, device="cuda").bfloat16() for _ in range(2))
    q = queries(c, "bf16")
    keep = {}
    stream = torch.cuda.Stream()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    n0 = lc.clone()
    pool0 = c.pool.clone()
    with torch.cuda.stream(stream):
        c.decode(q, "bf16", open_end=True, live=lc, k_tok=k, v_tok=v, counters=True, bins=9, stream=stream, keep=keep)
    stream.synchronize()
    lc.copy_(n0)
    c.pool.copy_(pool0)
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=stream):
        tg.tg_decode_mx(keep["args"], c.fmt, 0.0, stream)
    for step in range(4):
        k.normal_()
        v.normal_()
        q.normal_()
        torch.cuda.synchronize()
        graph.replay()
        out, lse, _ = e.decode(q, "bf16", open_end=True, live=le, k_tok=k, v_tok=v, counters=True, bins=9)
        torch.cuda.synchronize()
        assert torch.equal(keep["out"], out) and torch.equal(keep["lse"], lse)
        assert torch.equal(lc, le) and torch.equal(c.pool, e.pool) and int(keep["counters"].abs().sum()) == 0


def test_pages_past_32_bits():
    c = Cache([333, 20], H=8, gqa=2, d=128, Hp=8, bits=(8, 8))
    per = tg.tg_mx_page_bytes(c.geom, c.fmt)
    far = (1 << 32) // per + 50
    pool = torch.empty((far + c.pool_pages, 8, per // 8), dtype=torch.uint8, device="cuda")
    pool[far:] = c.pool
    q = queries(c, "bf16")
    near, lse, _ = c.decode(q, "bf16")
    c.pool, c.tables[0] = pool, c.tables[0] + far
    out, lse2, _ = c.decode(q, "bf16")
    assert torch.equal(near, out) and torch.equal(lse, lse2)
