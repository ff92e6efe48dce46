"""Quantised caches for the tests: tables from the library, bytes and attention from the 64-bit reference."""
import math

import numpy as np
import torch

from oracle import mx
from paper_2606_06302_amd import tangram as tg
from paper_2606_06302_amd.device import bind_decode, to_device, upload_plan

DTYPE = {"f32": torch.float32, "bf16": torch.bfloat16}
TG = {"f32": tg.TG_F32, "bf16": tg.TG_BF16}
FORMATS = [(4, 4), (8, 4), (4, 8), (8, 8)]


def fmt(bits):
    form = {4: tg.TG_MX_FP4, 8: tg.TG_MX_FP8}
    return tg.make_mx_format(form[bits[0]], form[bits[1]])


def f64(t):
    return t.double().cpu().numpy()


class Cache:
    """One batch's quantised pool: every retained row normal values, every other byte 0xff (scale bytes of NaN)."""

    def __init__(self, lens, H=4, gqa=2, d=64, Hp=2, bits=(4, 4), L=1, headroom=3, seed=0, fill=True, spare=5):
        rng = np.random.default_rng(seed)
        self.rng = rng
        self.B, self.H, self.L, self.d, self.Hp, self.bits, self.gqa = len(lens), H, L, d, Hp, bits, gqa
        self.geom = tg.tg_geometry(L, H, H * gqa, d, 16, Hp)
        self.fmt = fmt(bits)
        budget = rng.uniform(0.2, 1.0, (L, H))
        _, self.group_of, self.slot_of = tg.tg_cluster_heads(self.geom, budget)
        ctx = np.asarray(lens, np.int32)
        self.ratio = np.clip(budget[None] * rng.uniform(0.8, 1.0, (self.B, L, H)), 1e-6, 1.0)
        hr = np.full(self.B, headroom, np.int32)
        need = tg.tg_reserve(self.geom, ctx, self.ratio, None, self.group_of, np.zeros(0, np.int32), 0, size_query=True,
                             headroom=hr)["pages_needed"]
        self.pool_pages = need + spare
        free = rng.permutation(self.pool_pages).astype(np.int32)
        r = tg.tg_reserve(self.geom, ctx, self.ratio, None, self.group_of, free, self.pool_pages, headroom=hr)
        self.ctx, self.kv_len, self.offsets, self.pages = ctx, r["kv_len"], r["pt_offsets"], r["pt_pages"]
        self.places = mx.Places(d, *bits)
        assert tg.tg_mx_page_bytes(self.geom, self.fmt) == Hp * self.places.bytes
        self.host = np.full((self.pool_pages, Hp, self.places.bytes), 0xff, np.uint8)
        if fill:
            self._fill()
        self.tables = [to_device(a, "cuda") for a in (self.pages, self.offsets, self.group_of, self.slot_of)]
        self.pool = torch.from_numpy(self.host.copy()).cuda()

    def _fill(self):
        # random codes under scales within a few powers of two: as rows of normal values have them, at no cost
        for bits, byte, bit, scale in self.places.parts:
            for t in range(16):
                self.host[:, :, byte[t]] = self.rng.integers(0, 256, self.host[:, :, byte[t]].shape)
                if bits == 8:      # no code of NaN
                    x = self.host[:, :, byte[t]]
                    self.host[:, :, byte[t]] = np.where((x & 127) == 127, x - 1, x)
                self.host[:, :, scale[t]] = self.rng.integers(-3, 1, self.host[:, :, scale[t]].shape) + (125 if bits == 4 else 119)
        keep = np.zeros(self.host.shape[:2] + (16,), bool)
        for b, l, h in np.ndindex(self.B, self.L, self.H):
            page, slot = self.slabs(b, l, h, int(self.kv_len[b, l, h]))
            for i in range(int(self.kv_len[b, l, h])):
                keep[page[i // 16], slot, i % 16] = True
        clean = np.full_like(self.host, 0xff)
        for bits, byte, bit, scale in self.places.parts:
            for t in range(16):
                at = keep[:, :, t]
                for place in (np.unique(byte[t]), scale[t]):
                    x = clean[:, :, place]
                    x[at] = self.host[:, :, place][at]
                    clean[:, :, place] = x
        self.host = clean

    def slabs(self, b, l, h, n):
        """Page ids and the slot of the first n entries of a head."""
        G = self.H // self.Hp
        lo = int(self.offsets[(b * self.L + l) * G + self.group_of[l, h]])
        return self.pages[lo:lo + (n + 15) // 16], int(self.slot_of[l, h])

    def rows(self, b, l, h, n, host=None):
        page, slot = self.slabs(b, l, h, n)
        return [x[:n] for x in self.places.rows((self.host if host is None else host)[page, slot])]

    def store(self, b, l, h, entry, k, v):
        page, slot = self.slabs(b, l, h, entry + 1)
        self.places.store(self.host[page[-1], slot], entry % 16, k, v)

    # ---------------------------------------------------------------- decode
    def decode(self, q, dtype, layer=0, softcap=0.0, sm_scale=0.0, bins=None, mode=tg.TG_PLAN_AOT_FILL, open_end=False,
               live=None, k_tok=None, v_tok=None, counters=False, full=None, timestamps=None, stream=None, keep=None):
        """-> out, lse tensors of one call."""
        g = self.geom
        if bins is None:
            bins = tg.tg_decode_mx_bins(g, TG[dtype], self.fmt, 0, self.B, layer, self.kv_len)
        plan = tg.tg_build_plan(g, self.B, layer, self.kv_len, self.offsets, self.group_of, self.slot_of,
                                mode | (tg.TG_PLAN_OPEN_END if open_end else 0), bins, split_target=bins)
        dp = upload_plan(g, self.B, plan, "cuda")
        out = torch.full_like(q, float("nan"))
        lse = torch.full(q.shape[:2], float("nan"), dtype=torch.float32, device="cuda")
        cnt = torch.zeros(self.B * self.H, dtype=torch.int32, device="cuda") if counters else None
        args = bind_decode(dp, g, self.B, TG[dtype], q, self.pool, self.tables[0], out, lse, sm_scale=sm_scale,
                           live_len=live, layer=layer, merge_counters=cnt)
        if k_tok is not None:
            args.append_k, args.append_v = k_tok.data_ptr(), v_tok.data_ptr()
        if full is not None:
            args.append_full = full.data_ptr()
        if timestamps is not None:
            args.timestamps = timestamps.data_ptr()
        if keep is not None:
            keep.update(args=args, plan=dp, counters=cnt, out=out, lse=lse)
        tg.tg_decode_mx(args, self.fmt, softcap, stream)
        if keep is None:
            torch.cuda.synchronize()
            assert cnt is None or int(cnt.abs().sum()) == 0
        return out, lse, plan


def attend(q, k, v, scale, cap):
    """out [d], lse, and the sizes that bound what rounding may do: sum p |v| [d], the largest sum |q k| scale."""
    z = k @ q * scale
    if cap > 0:
        z = cap * np.tanh(z / cap)
    top = z.max()
    p = np.exp(z - top)
    total = p.sum()
    p = p / total
    return p @ v, top + math.log(total), p @ np.abs(v), float((np.abs(k) @ np.abs(q)).max()) * scale


def check_decode(c, q, out, lse, dtype, layer=0, softcap=0.0, sm_scale=0.0, lens=None, host=None, what=""):
    """Every head against 64 bits.  K and V are exact and so are their products with q in fp32; what rounds:
      * a score: d products summed in fp32, each step off by 2^-23 of the sizes summed (the matrix cores may cut): d 2^-23
        of sum |q k|, once more the scaling, and the cap's 6e-7 |s| (at most of the same sum);
      * a weight: 2^-21 for the exponential and its argument, and in bf16 calls half a step of bf16, 2^-8;
      * the sums over n weights: n 2^-23 of sum p |v|;
      * the result: half a step of its type, 2^-8 of it in bf16 (2^-22 for the division in fp32)."""
    scale = sm_scale if sm_scale else 1 / math.sqrt(c.d)
    lens = c.kv_len[:, layer] if lens is None else lens
    qh, o, ls = f64(q), f64(out), f64(lse)
    worst = 0.0
    for b in range(c.B):
        for h in range(c.H):
            n = int(lens[b, h])
            k, v = c.rows(b, layer, h, n, host)
            for j in range(h * c.gqa, (h + 1) * c.gqa):
                want, wl, size, qk = attend(qh[b, j], k, v, scale, softcap)
                score = qk * (c.d * 2.0 ** -23 + 2.0 ** -23 + (6e-7 if softcap else 0.0))
                weight = 2 * score + 2.0 ** -21 + n * 2.0 ** -23
                half = 2.0 ** -8 if dtype == "bf16" else 2.0 ** -22
                bound = size * (weight + (2.0 ** -8 if dtype == "bf16" else 0.0)) * 1.01 + np.abs(want) * half + 1e-37
                off = np.abs(o[b, j] - want)
                assert np.all(off <= bound), f"{what} b {b} head {j} n {n}: off {(off / bound).max():.2f} times the bound"
                assert abs(ls[b, j] - wl) <= weight + 2.0 ** -21 * (1 + abs(wl)), f"{what} b {b} head {j}: lse off {abs(ls[b, j] - wl)}"
                worst = max(worst, float((off / bound).max()))
    return worst
