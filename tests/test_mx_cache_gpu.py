"""A quantised cache: what append, compression and read-back store and return, byte for byte."""
import numpy as np
import pytest
import torch

import oracle
from gpu_helpers import say

pytestmark = pytest.mark.gpu

if torch.cuda.is_available():
    from mx_helpers import DTYPE, FORMATS, TG, Cache, f64, fmt
    from oracle import mx
    from paper_2606_06302_amd import tangram as tg
    from paper_2606_06302_amd.device import to_device
else:
    FORMATS = [(4, 4), (8, 4), (4, 8), (8, 8)]


@pytest.fixture(autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def hard_rows(n, d, dtype, rng):
    """Rows with what quantisation can go wrong at: ties, sizes at a scale's border, signed zeros, tiny and huge values,
    denormal numbers, NaN and infinities, and ordinary rows between them."""
    first = np.arange(d) % 32 == 5                       # one element of every group
    past = lambda x: np.nextafter(np.float32(x), np.float32(2 * x))
    kinds = [lambda r: r, lambda r: r * 0.0, lambda r: r * -0.0, lambda r: np.round(r * 8) / 8,
             lambda r: np.round(r * 512) / 512, lambda r: np.clip(r * 1e38, -3e38, 3e38), lambda r: r * 1e-38,
             lambda r: r * 1e-41, lambda r: np.full(d, 1e-45), lambda r: np.full(d, 3.38e38),
             lambda r: r * 2.0 ** int(rng.integers(-110, 110)), lambda r: np.where(first, 7.0, r),
             lambda r: np.where(first, past(7), r), lambda r: np.where(first, 464.0, r), lambda r: np.where(first, past(464), r),
             lambda r: np.where(first, 1e30, r * 1e-30), lambda r: np.where(np.arange(d) == 40, np.nan, r),
             lambda r: np.where(np.arange(d) == 3, -np.inf, r)]
    x = np.stack([kinds[i % len(kinds)](rng.standard_normal(d)) for i in range(n)])
    return torch.from_numpy(x.astype(np.float32)).to(DTYPE[dtype]).cuda()


@pytest.mark.parametrize("bits", FORMATS)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d,H,Hp", [(128, 4, 2), (64, 3, 1)])
def test_append_stores_the_reference_bytes(bits, dtype, d, H, Hp):
    c = Cache([1, 15, 16, 17, 33, 70], H=H, d=d, Hp=Hp, bits=bits, L=2, headroom=4, seed=d + H)
    layer = 1
    live = to_device(c.kv_len, "cuda")
    rng = np.random.default_rng(3)
    n = c.kv_len.copy()
    for step in range(3):
        k, v = (hard_rows(c.B * H, d, dtype, rng).view(c.B, H, d) for _ in range(2))
        args = tg.make_append_args(c.geom, c.B, layer, TG[dtype], k, v, c.pool, *c.tables, live)
        tg.tg_append_mx(args, c.fmt)
        for b, h in np.ndindex(c.B, H):
            c.store(b, layer, h, int(n[b, layer, h]), f64(k)[b, h], f64(v)[b, h])
        n[:, layer] += 1
        assert np.array_equal(live.cpu().numpy(), n)
        got = c.pool.cpu().numpy()
        assert np.array_equal(got, c.host), f"step {step}: {np.argwhere(got != c.host)[:4].tolist()}"


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_append_to_a_full_or_missing_table(dtype):
    c = Cache([16, 20], H=2, d=64, Hp=1, headroom=2)
    capacity = np.diff(c.offsets).reshape(2, 2)[:, c.group_of[0]] * 16      # [request][head]
    n = c.kv_len.copy()
    n[0, 0] = capacity[0]                                                   # both heads full
    n[1, 0, 0] = -1                                                         # no length
    live, full = to_device(n, "cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    k, v = (torch.randn(2, 2, 64, device="cuda").to(DTYPE[dtype]) for _ in range(2))
    tg.tg_append_mx(tg.make_append_args(c.geom, 2, 0, TG[dtype], k, v, c.pool, *c.tables, live, full), c.fmt)
    c.store(1, 0, 1, int(n[1, 0, 1]), f64(k)[1, 1], f64(v)[1, 1])
    n[1, 0, 1] += 1
    assert int(full) == 1 and np.array_equal(live.cpu().numpy(), n) and np.array_equal(c.pool.cpu().numpy(), c.host)
    # a group id out of range has no table
    full.zero_()
    bad = torch.full_like(c.tables[2], 9)
    tg.tg_append_mx(tg.make_append_args(c.geom, 2, 0, TG[dtype], k, v, c.pool, c.tables[0], c.tables[1], bad, c.tables[3],
                                        live, full), c.fmt)
    assert int(full) == 1 and np.array_equal(live.cpu().numpy(), n) and np.array_equal(c.pool.cpu().numpy(), c.host)


@pytest.mark.parametrize("bits", FORMATS)
@pytest.mark.parametrize("dtype,d,C", [("bf16", 128, 1), ("bf16", 128, 130), ("f32", 64, 97), ("bf16", 64, 1100),
                                       ("f32", 128, 1030)])
def test_compress_stores_the_kept_rows(bits, dtype, d, C):
    H, B = 4, 3
    rng = np.random.default_rng(C + d)
    before = np.array([0, 37, 5], np.int32)
    valid = np.array([C, max(1, C // 2), C], np.int32)
    c = Cache(before + valid, H=H, d=d, Hp=2, bits=bits, seed=C, headroom=0)
    k, v = (hard_rows(B * C * H, d, dtype, rng).view(B, C, H, d) for _ in range(2))
    scores = torch.from_numpy((np.round(rng.standard_normal((B, H, C)) * 16) / 16).astype(np.float32)).cuda()
    plan = tg.tg_compress_plan(c.geom, B, 0, C, before, valid, c.ratio, None, c.kv_len, c.offsets, c.group_of, c.slot_of,
                               rows_per_item=23)
    kept = torch.full((B, H, C), -1, dtype=torch.int32, device="cuda")
    items = to_device(plan["items"] if plan["num_items"] else np.zeros(1, tg.COMPRESS_ITEM_DTYPE), "cuda")
    args = tg.make_compress_args(c.geom, B, C, TG[dtype], k, v, scores, c.pool, c.tables[0], items, plan["num_items"],
                                 to_device(valid, "cuda"), to_device(plan["keep_count"], "cuda"), kept)
    tg.tg_compress_mx(args, c.fmt)
    got_kept, sc, kh, vh = kept.cpu().numpy(), scores.cpu().numpy(), f64(k), f64(v)
    for b, h in np.ndindex(B, H):
        n = int(plan["keep_count"][b, h])
        best = np.sort(oracle.top_entries(sc[b, h, :valid[b]].astype(np.float64), n))
        assert np.array_equal(got_kept[b, h, :n], best) and np.all(got_kept[b, h, n:] == -1)
        for j, t in enumerate(best):
            c.store(b, 0, h, int(plan["write_begin"][b, h]) + j, kh[b, t, h], vh[b, t, h])
    got = c.pool.cpu().numpy()
    assert np.array_equal(got, c.host), np.argwhere(got != c.host)[:4].tolist()


@pytest.mark.parametrize("bits", FORMATS)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d,H,Hp", [(128, 4, 2), (64, 6, 3)])
def test_unpack_returns_what_the_codes_stand_for(bits, dtype, d, H, Hp):
    c = Cache([1, 16, 17, 70, 300], H=H, d=d, Hp=Hp, bits=bits, L=2, seed=7 * d)
    layer = 1
    # one row of NaN codes, and lengths past the capacity, are part of it
    c.host[c.slabs(3, layer, 0, 1)[0][0], c.slot_of[layer, 0], c.places.parts[0][3][0]] = 255
    c.pool.copy_(torch.from_numpy(c.host))
    G = H // Hp
    rows = torch.full((c.pool_pages, 2, Hp, 16, d), 77.0, dtype=DTYPE[dtype], device="cuda")
    want = f64(rows)
    begin = np.minimum(c.kv_len - 1, np.arange(c.B)[:, None, None] * 9).astype(np.int32)
    begin[1] = -5
    args = tg.make_unpack_mx_args(c.geom, c.B, layer, TG[dtype], c.fmt, c.pool, *c.tables, to_device(c.kv_len, "cuda"), rows,
                                  begin=to_device(begin, "cuda"))
    tg.tg_unpack_mx(args)
    for b, h in np.ndindex(c.B, H):
        n, lo = int(c.kv_len[b, layer, h]), max(0, int(begin[b, layer, h]))
        page, slot = c.slabs(b, layer, h, n)
        for i, x in enumerate(c.rows(b, layer, h, n)):
            for e in range(lo, n):
                want[page[e // 16], i, slot, e % 16] = x[e]
    got = f64(rows)
    assert np.array_equal(got, want, equal_nan=True), np.argwhere((got != want) & ~np.isnan(want))[:4].tolist()
    # the same into a layer's own pages, from the start, with lengths that say too much
    tables = np.arange(len(c.offsets) - 1).reshape(c.B, c.L, G)[:, layer].reshape(-1)
    dst, at = np.full(len(c.pages), -1, np.int32), 0
    for t in tables:
        m = int(c.offsets[t + 1] - c.offsets[t])
        dst[c.offsets[t]:c.offsets[t + 1]] = np.arange(at, at + m)
        at += m
    small = torch.full((at, 2, Hp, 16, d), 77.0, dtype=DTYPE[dtype], device="cuda")
    args = tg.make_unpack_mx_args(c.geom, c.B, layer, TG[dtype], c.fmt, c.pool, *c.tables,
                                  torch.full((c.B, c.L, H), 1 << 30, dtype=torch.int32, device="cuda"), small,
                                  dst_pages=to_device(dst, "cuda"))
    tg.tg_unpack_mx(args)
    got = f64(small)
    for b, h in np.ndindex(c.B, H):
        t = (b * c.L + layer) * G + int(c.group_of[layer, h])
        ids, slot = c.pages[c.offsets[t]:c.offsets[t + 1]], int(c.slot_of[layer, h])
        for i, x in enumerate(c.places.rows(c.host[ids, slot])):
            assert np.array_equal(got[dst[c.offsets[t]:c.offsets[t + 1]], i, slot].reshape(-1, d), x, equal_nan=True)


def test_unpack_of_nothing():
    c = Cache([40, 9], H=2, d=64, Hp=1)
    rows = torch.full((c.pool_pages, 2, 1, 16, 64), 5.0, device="cuda")
    for length in (0, -3):
        args = tg.make_unpack_mx_args(c.geom, 2, 0, tg.TG_F32, c.fmt, c.pool, *c.tables,
                                      torch.full((2, 1, 2), length, dtype=torch.int32, device="cuda"), rows)
        tg.tg_unpack_mx(args)
    assert bool((rows == 5.0).all())


def test_every_code_reads_back():
    """All codes under all scales that the quantiser gives, both parts, both types."""
    for bits in (4, 8):
        c = Cache([16 * 253], H=1, gqa=1, d=64, Hp=1, bits=(bits, bits), headroom=0, fill=False)
        n = int(c.kv_len[0, 0, 0])
        rng = np.random.default_rng(bits)
        lo, hi = mx.RANGE[bits]
        slabs = rng.integers(0, 256, c.host.shape).astype(np.uint8)
        for part, (_, byte, bit, scale) in enumerate(c.places.parts):
            if bits == 8:
                slabs[..., byte.reshape(-1)] = np.where((slabs[..., byte.reshape(-1)] & 127) == 127, 0, slabs[..., byte.reshape(-1)])
            slabs[..., scale.reshape(-1)] = rng.integers(lo + 127, hi + 128, slabs[..., scale.reshape(-1)].shape)
        c.pool.copy_(torch.from_numpy(slabs))
        for dtype in ("bf16", "f32"):
            rows = torch.zeros(c.pool_pages, 2, 1, 16, 64, dtype=DTYPE[dtype], device="cuda")
            tg.tg_unpack_mx(tg.make_unpack_mx_args(c.geom, 1, 0, TG[dtype], c.fmt, c.pool, *c.tables,
                                                   to_device(c.kv_len, "cuda"), rows))
            page, slot = c.slabs(0, 0, 0, n)
            for i, want in enumerate(c.rows(0, 0, 0, n, slabs)):
                assert np.array_equal(f64(rows)[page, i, slot].reshape(-1, 64)[:n], want)
        say(f"bits {bits}: {n} rows")


def test_pool_past_32_bits():
    """Pages whose bytes lie past 4 GiB, on a stream of their own."""
    c = Cache([33, 5], H=8, gqa=1, d=128, Hp=8, bits=(8, 8), headroom=2)
    per = tg.tg_mx_page_bytes(c.geom, c.fmt)
    far = (1 << 32) // per + 50
    pool = torch.empty((far + c.pool_pages, 8, per // 8), dtype=torch.uint8, device="cuda")
    pool[far:] = c.pool
    pages = c.tables[0] + far
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    live = to_device(c.kv_len, "cuda")
    k, v = (torch.randn(2, 8, 128, device="cuda").bfloat16() for _ in range(2))
    rows = torch.zeros(c.pool_pages, 2, 8, 16, 128, dtype=torch.bfloat16, device="cuda")
    torch.cuda.synchronize()
    tg.tg_append_mx(tg.make_append_args(c.geom, 2, 0, tg.TG_BF16, k, v, pool, pages, *c.tables[1:], live), c.fmt, stream)
    tg.tg_unpack_mx(tg.make_unpack_mx_args(c.geom, 2, 0, tg.TG_BF16, c.fmt, pool, pages, *c.tables[1:], live, rows,
                                           dst_pages=c.tables[0]), stream)
    stream.synchronize()
    for b, h in np.ndindex(2, 8):
        c.store(b, 0, h, int(c.kv_len[b, 0, h]), f64(k)[b, h], f64(v)[b, h])
    assert np.array_equal(pool[far:].cpu().numpy(), c.host)
    for b, h in np.ndindex(2, 8):
        n = int(c.kv_len[b, 0, h]) + 1
        page, slot = c.slabs(b, 0, h, n)
        for i, want in enumerate(c.rows(b, 0, h, n)):
            assert np.array_equal(f64(rows)[page, i, slot].reshape(-1, 128)[:n], want)
    del pool
