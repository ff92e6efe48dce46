"""tg_prefill_mod and tg_decode_capped against a plain 64-bit form.

Tolerance of an output, with W = sum_k p_k |v_k| / sum_k p_k in 64 bits:
  bf16: 2^-8 |o| (the result's rounding) + 2^-8 W (the probabilities', head_dim 64 decode keeps more) + 1e-3 W: an error
    e of a score multiplies its probability by 1 + e, in the numerator and the sum; the scores are fp32 sums of at most
    128 products, 2^-24 * 136 * A of error for A = sm_scale * sum |q_i k_i|, at most 40 here (3.3e-4), and the cap adds
    6e-7 of a score at most 1000 in the cases (below 2e-4 with |s| <= 300): twice their sum stays below 1.1e-3.
  f32: 2^-23 |o| + (2e-5 + 2 (1e-6 A + 3e-7 cap)) W: chains of at most 200 roundings of 2^-24 in the long sums
    (1.2e-5), the exponentials and the weights that join waves and pieces (a few 1e-7 each), the scores as above in
    trees of at most 16 roundings.
"""
import math

import numpy as np
import pytest
import torch

from gpu_helpers import poisoned_host_pool, say
from workloads import Geometry, custom

pytestmark = pytest.mark.gpu

if torch.cuda.is_available():
    from paper_2606_06302_amd import tangram as tg
    from paper_2606_06302_amd.runner import DecodeSession, PrefillSession, Tables


def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def cuda(a, dtype=np.int32):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=dtype)).cuda()


def host_rows(pool, t, g, b, layer, h, n):
    """K and V rows [n][d] of head (b, layer, h), float64, from the pool on the host."""
    base = int(t.pt_offsets[(b * g.num_layers + layer) * g.num_groups + int(t.group_of[layer, h])])
    ids = t.pt_pages[base:base + -(-n // g.page_size)]
    kv = pool[ids][:, :, int(t.slot_of[layer, h])]
    return (kv[:, i].reshape(-1, g.head_dim)[:n] for i in (0, 1))


def attend(q, k, v, seen, scale, cap):
    """(out, W) of rows q [n][d] over keys k, v [m][d] where seen [n][m]; zeros where a row sees nothing."""
    with np.errstate(all="ignore"):
        s = (q @ k.T) * scale
        if cap > 0:
            s = cap * np.tanh(s / cap)
        s = np.where(seen, s, -np.inf)
        m = s.max(1, keepdims=True, initial=-np.inf)
        p = np.where(seen, np.exp(s - np.where(np.isfinite(m), m, 0)), 0)
        z = p.sum(1, keepdims=True)
        p = p / np.where(z > 0, z, 1)
        v0 = np.where(seen.any(0)[:, None], v, 0)          # rows that nobody sees may hold anything
        return p @ v0, p @ np.abs(v0)


def f64(x):
    return x.float().cpu().numpy().astype(np.float64)


# --------------------------------------------------------------------- prefill
def masks(kind, rng, B, C, tokens):
    """(key_begin, key_end) arrays [B][C] or None, None."""
    if kind == "causal":
        return None, None
    at = np.tile(np.arange(C), (B, 1))
    if kind == "prefix":
        return None, np.maximum(at + 1, rng.integers(0, C + 1, (B, 1)))
    if kind == "bidirectional":
        return np.full((B, C), -7), np.full((B, C), 2 ** 31 - 1)
    if kind == "documents":
        begin = np.full((B, C), -1)
        for b in range(B):
            for c in np.sort(rng.integers(0, C, 3)):
                begin[b, c:] = c
        return begin, None
    if kind == "window":
        return np.maximum(at + 1 - max(1, C // 3), 0), None
    # any ranges: rows without a key, without the history, starting anywhere
    begin = rng.integers(-C // 2 - 1, C, (B, C))
    end = begin + rng.integers(-3, C + 2, (B, C))
    blank = rng.random((B, C)) < 0.2
    begin, end = np.where(blank, 0, begin), np.where(blank, -2 ** 31, end)
    begin[0, :C // 2], end[0, :C // 2] = 2 ** 31 - 1, 0          # whole waves of rows without a key
    return begin, end


class Prefill:
    def __init__(self, seed, H, gqa, d, Hp, B, C, ctx, mask, cap, q_scale=1.0, tokens=None, hist=None, split=None,
                 schedule=True, nan=True):
        rng = np.random.default_rng(seed)
        g = Geometry(2, H, H * gqa, d, 16, Hp)
        self.wl = custom(seed, g, B, "bf16", ctx, chunk_len=C, q_scale=q_scale, kv_scale=0.7)
        self.t = Tables(self.wl)
        self.layer, self.cap, self.C = 1, cap, C
        self.tokens = None if tokens is None else np.asarray(tokens)
        self.begin, self.end = masks(mask, rng, B, C, tokens)
        pool = torch.from_numpy(poisoned_host_pool(self.wl, self.t)).bfloat16()
        self.keep = [None if x is None else cuda(np.clip(x, -2 ** 31, 2 ** 31 - 1)) for x in (self.tokens, self.begin, self.end)]
        mod = tg.make_score_mod(cap, *self.keep)
        self.hist = self.t.kv_len if hist is None else np.minimum(self.t.kv_len, hist).astype(np.int32)
        self.s = PrefillSession(self.wl, tables=self.t, layer=1, fill="host", pool=pool.cuda(), hist_len=self.hist, mod=mod,
                                schedule=schedule)
        a = self.s.args
        need = tg.tg_prefill_workspace_bytes(a)
        if split is True:
            self.ws = torch.full((need,), 0x7F, dtype=torch.uint8, device="cuda")    # fp32 NaN-ish bytes
            a.workspace, a.workspace_bytes = self.ws.data_ptr(), need
        elif split is False:
            a.workspace, a.workspace_bytes = None, 0
        if nan and self.tokens is not None:
            for b, n in enumerate(self.tokens):
                for x in (self.s.q, self.s.k_new, self.s.v_new):
                    x[b, max(0, int(n)):] = float("nan")
        self.s.out.fill_(float("nan"))
        self.pool = f64(self.s.pool)

    def seen(self, b):
        """[C][C] chunk keys each row sees, [C] whether it sees the history, [C] valid rows."""
        C = self.C
        n = C if self.tokens is None else min(max(int(self.tokens[b]), 0), C)
        at = np.arange(C)
        begin = np.full(C, -1) if self.begin is None else self.begin[b]
        end = at + 1 if self.end is None else self.end[b]
        return (at[None] >= begin[:, None]) & (at[None] < np.minimum(end, n)[:, None]), begin < 0, at < n

    def check(self, what):
        g, s = self.wl.geom, self.s
        got, q, kn, vn = f64(s.out), f64(s.q), f64(s.k_new), f64(s.v_new)
        scale = 1 / math.sqrt(g.head_dim)
        worst = 0.0
        for b in range(self.wl.batch):
            chunk, hist, valid = self.seen(b)
            for h in range(g.num_kv_heads):
                n = int(self.hist[b, self.layer, h])
                k, v = host_rows(self.pool, self.t, g, b, self.layer, h, n)
                k, v = np.concatenate([k, kn[b, :, h]]), np.concatenate([v, vn[b, :, h]])
                vis = np.concatenate([np.tile(hist[:, None], (1, n)), chunk], 1)[valid]
                for j in range(h * g.gqa, (h + 1) * g.gqa):
                    o, w = attend(q[b, valid, j], k, v, vis, scale, self.cap)
                    assert np.all(np.isnan(got[b, ~valid, j])), (what, "rows past the request's tokens were written")
                    gj = got[b, valid, j]
                    tol = 2.0 ** -8 * np.abs(o) + (2.0 ** -8 + 1e-3) * w
                    assert np.all(np.isfinite(gj)), (what, b, j)
                    assert not gj[~vis.any(1)].any(), (what, "a row without keys")
                    over = np.abs(gj - o) - tol
                    assert over.max(initial=-1) <= 1e-30, (what, b, j, float(over.max()), np.unravel_index(over.argmax(), over.shape))
                    ok = tol > 0
                    worst = max(worst, float((np.abs(gj - o)[ok] / tol[ok]).max(initial=0)))
        say(f"{what}: {worst:.2f} of the tolerance")


SHAPES = [  # H, gqa, d, Hp, B, C, ctx, tokens
    (2, 4, 128, 2, 2, 65, (40, 300), None), (4, 1, 64, 2, 2, 130, (100, 700), [130, 77]),
    (2, 16, 128, 1, 1, 33, 500, None), (2, 5, 64, 2, 3, 100, (1, 90), [0, 100, 1]),
    (2, 7, 128, 2, 3, 1, 64, [1, 0, 1]), (1, 8, 64, 1, 1, 257, 33, [200]), (2, 3, 128, 2, 2, 300, (700, 900), [299, 64])]


@pytest.mark.parametrize("mask", ["causal", "prefix", "bidirectional", "documents", "window", "any"])
@pytest.mark.parametrize("cap", [0.0, 5.0])
@pytest.mark.parametrize("split", [False, True])
@pytest.mark.parametrize("H,gqa,d,Hp,B,C,ctx,tokens", SHAPES)
def test_prefill_masks_and_caps(mask, cap, split, H, gqa, d, Hp, B, C, ctx, tokens):
    _gpu()
    p = Prefill(100 + C + d, H, gqa, d, Hp, B, C, ctx, mask, cap, tokens=tokens, split=split)
    p.s.run()
    torch.cuda.synchronize()
    p.check(f"prefill {mask} cap {cap} split {split}")


@pytest.mark.parametrize("cap,q_scale", [(50.0, 3.0), (1.0, 10.0), (1000.0, 1.0), (30.0, 8.0), (0.01, 4.0), (1e-3, 1.0), (1e6, 2.0)])
@pytest.mark.parametrize("d", [64, 128])
def test_prefill_caps_from_far_below_to_far_above_the_scores(cap, q_scale, d):
    _gpu()
    for split in (False, True):
        p = Prefill(7, 2, 4, d, 2, 2, 70, (200, 400), "causal", cap, q_scale=q_scale, split=split)
        p.s.run()
        torch.cuda.synchronize()
        p.check(f"prefill cap {cap} scale {q_scale} split {split}")


@pytest.mark.parametrize("split", [False, True])
@pytest.mark.parametrize("d", [64, 128])
def test_prefill_without_history(split, d):
    _gpu()
    for mask in ("causal", "any", "documents"):
        p = Prefill(8, 2, 4, d, 2, 2, 90, 50, mask, 0.0, hist=0, split=split)
        p.s.run()
        torch.cuda.synchronize()
        p.check(f"no history {mask} {split}")


@pytest.mark.parametrize("d", [64, 128])
def test_prefill_longer_history_with_the_pieces_of_few_blocks(d):
    """One request whose blocks are cut into many pieces, some of which hold only keys that some rows do not see."""
    _gpu()
    for mask, cap in (("documents", 20.0), ("any", 0.0), ("prefix", 0.0), ("causal", 50.0)):
        p = Prefill(9, 2, 8, d, 2, 1, 150, 6000, mask, cap, q_scale=2.0, split=True)
        p.s.run()
        torch.cuda.synchronize()
        p.check(f"pieces {mask}")


@pytest.mark.parametrize("d,gqa", [(128, 4), (64, 5)])
def test_no_mask_no_cap_is_tg_prefill(d, gqa):
    """Neither a cap nor a mask: tg_prefill's output bit for bit, whatever the block order (whole blocks; the key-split
    launches cut in different places)."""
    _gpu()
    p = Prefill(10, 4, gqa, d, 2, 3, 200, (300, 3000), "causal", 0.0, split=False)
    p.s.run()
    got = p.s.out.clone()
    p.s.out.fill_(float("nan"))
    tg.tg_prefill(p.s.args)
    torch.cuda.synchronize()
    assert torch.equal(got, p.s.out)
    p.s.out.fill_(float("nan"))
    p.s.args.block_order, p.s.args.num_blocks = None, 0
    p.s.run()
    torch.cuda.synchronize()
    assert torch.equal(got, p.s.out)


@pytest.mark.parametrize("split", [False, True])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("bad", [float("inf"), -float("inf"), float("nan")])
def test_what_a_row_does_not_see_does_not_reach_it(split, d, bad):
    """Keys and values of one document, and of the history that it alone sees, hold infinities or NaN: the other
    document's rows are those of finite inputs, bit for bit; visible ones come through as the formula has them."""
    _gpu()
    p = Prefill(11, 2, 4, d, 2, 1, 96, 200, "causal", 0.0, split=split)
    begin = np.full((1, 96), -1)
    begin[0, 50:] = 50                       # tokens 50.. see neither the history nor tokens 0..49
    p.keep[1] = cuda(begin)
    p.s.mod.key_begin = p.keep[1].data_ptr()
    p.begin = begin
    p.s.run()
    torch.cuda.synchronize()
    p.check("finite")
    clean = p.s.out.clone()
    p.s.k_new[0, 10] = bad
    p.s.v_new[0, 20, 0] = bad
    p.s.v_new[0, 49, :, 3] = bad
    p.s.run()
    torch.cuda.synchronize()
    assert torch.equal(p.s.out[0, 50:], clean[0, 50:])
    # token 10's key is seen by tokens 10..49 alone: rows before it are clean; a NaN score makes the row NaN, an
    # infinite one too (its sign differs by dim, so its products cancel to NaN)
    assert torch.equal(p.s.out[0, :10], clean[0, :10])
    assert bool(torch.isnan(p.s.out[0, 10:50]).all())
    # values alone: row 20 and later of head 0 take the value itself, row 49 of dim 3 in every head
    p.s.k_new[0, 10] = 0.5
    p.s.v_new[0, 20, 0], p.s.v_new[0, 49, :, 3] = 0.25, 0.25
    p.s.run()
    torch.cuda.synchronize()
    clean = p.s.out.clone()
    p.s.v_new[0, 20, 0] = bad
    p.s.v_new[0, 49, 1, 3] = bad
    p.s.run()
    torch.cuda.synchronize()
    o = p.s.out
    gqa = 4
    assert torch.equal(o[0, :20], clean[0, :20]) and torch.equal(o[0, 50:], clean[0, 50:])
    want = torch.full_like(o[0, 20:50, :gqa], bad)
    assert torch.equal(o[0, 20:50, :gqa].nan_to_num(7, 8, 9), want.nan_to_num(7, 8, 9))
    assert torch.equal(o[0, 20:49, gqa:], clean[0, 20:49, gqa:])
    assert bool((o[0, 49, gqa:, 3].nan_to_num(7, 8, 9) == torch.tensor(bad).bfloat16().nan_to_num(7, 8, 9).item()).all())
    keep = [e for e in range(d) if e != 3]
    assert torch.equal(o[0, 49, gqa:][:, keep], clean[0, 49, gqa:][:, keep])


def test_history_that_only_some_rows_see_may_hold_infinities():
    _gpu()
    for d in (64, 128):
        p = Prefill(12, 1, 4, d, 1, 1, 40, 100, "causal", 0.0, split=False)
        begin = np.where(np.arange(40) % 2 == 0, -1, 0)[None]
        p.keep[1] = cuda(begin)
        p.s.mod.key_begin = p.keep[1].data_ptr()
        p.s.run()
        torch.cuda.synchronize()
        clean = p.s.out.clone()
        base = int(p.t.pt_offsets[1 * 1 + 0])                        # layer 1's only table
        page = int(p.t.pt_pages[base])
        p.s.pool[page, 1, 0, 3, 5] = float("inf")
        p.s.run()
        torch.cuda.synchronize()
        assert torch.equal(p.s.out[0, 1::2], clean[0, 1::2])
        assert bool(torch.isinf(p.s.out[0, 0::2, :, 5]).all())
        rest = [e for e in range(d) if e != 5]
        assert torch.equal(p.s.out[0, 0::2][..., rest], clean[0, 0::2][..., rest])


@pytest.mark.parametrize("split", [False, True])
@pytest.mark.parametrize("d", [64, 128])
def test_infinite_scores_are_capped(d, split):
    """Scores of +-infinity are +-softcap: also where they are the first that a row sees, or all that it sees."""
    _gpu()
    for mask, cap in (("causal", 2.0), ("bidirectional", 4.0), ("documents", 1.0), ("any", 3.0), ("causal", 200.0)):
        p = Prefill(13, 1, 4, d, 1, 1, 100, 70, mask, cap, hist=0, split=split)
        p.s.q[..., 0] = 1.0
        p.s.k_new[0, :40, 0, 0] = -float("inf")
        p.s.k_new[0, 70, 0, 0] = float("inf")
        p.s.run()
        torch.cuda.synchronize()
        p.check(f"infinite scores {mask} cap {cap} split {split}")


def test_prefill_graph_and_streams():
    """Two captured calls with workspaces of their own, replayed side by side with new inputs, against the eager call."""
    _gpu()
    runs = []
    for seed in (13, 14):
        p = Prefill(seed, 2, 4, 128, 2, 2, 90, 2000, "documents", 30.0, tokens=[90, 41], split=True)
        st = torch.cuda.Stream()
        st.wait_stream(torch.cuda.current_stream())
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=st):
            p.s.run(st)
        runs.append((p, st, graph))
    for i in range(4):
        for p, st, graph in runs:
            p.s.q[:, :41].normal_()
        torch.cuda.synchronize()
        for p, st, graph in runs:
            with torch.cuda.stream(st):
                graph.replay()
        torch.cuda.synchronize()
        for p, st, graph in runs:
            got = p.s.out.clone()
            p.s.run(torch.cuda.current_stream())
            torch.cuda.synchronize()
            assert torch.equal(got.nan_to_num(1e9), p.s.out.nan_to_num(1e9)), i


@pytest.mark.parametrize("split", [False, True])
@pytest.mark.parametrize("d", [64, 128])
def test_pages_past_32_bits(d, split):
    """The same cache at the end of a pool of more than 2^32 bytes."""
    _gpu()
    p = Prefill(15, 2, 4, d, 1, 2, 70, 300, "documents", 10.0, split=split)
    p.s.run()
    torch.cuda.synchronize()
    near = p.s.out.clone()
    n, page = p.s.pool.shape[0], p.s.pool[0].numel() * 2
    shift = (2 ** 32 + 2 ** 20) // page
    pool = torch.empty(n + shift, *p.s.pool.shape[1:], dtype=torch.bfloat16, device="cuda")
    pool[shift:].copy_(p.s.pool)
    pages = p.t.d_pt_pages + shift
    p.s.args.kv_pool, p.s.args.pt_pages = pool.data_ptr(), pages.data_ptr()
    p.s.out.fill_(float("nan"))
    p.s.run()
    torch.cuda.synchronize()
    assert torch.equal(p.s.out, near)


# ---------------------------------------------------------------------- decode
def check_decode(s, cap, what):
    g, t, wl = s.wl.geom, s.t, s.wl
    scale = 1 / math.sqrt(g.head_dim)
    pool = f64(s.pool)
    live = t.kv_len if s.live_len is None else s.live_len.cpu().numpy()
    worst = 0.0
    for l in s.layers:
        q, out, lse = f64(s.q[l]), f64(s.out[l]), s.lse[l].double().cpu().numpy()
        for b in range(wl.batch):
            for h in range(g.num_kv_heads):
                n = int(live[b, l, h])
                k, v = host_rows(pool, t, g, b, l, h, n)
                rows = slice(h * g.gqa, (h + 1) * g.gqa)
                o, w = attend(q[b, rows], k, v, np.ones((g.gqa, n), bool), scale, cap)
                sc = cap * np.tanh(q[b, rows] @ k.T * scale / cap)
                m = sc.max(1, keepdims=True)
                ref = (m + np.log(np.exp(sc - m).sum(1, keepdims=True)))[:, 0]
                A = float((np.abs(q[b, rows]) @ np.abs(k).T).max()) * scale
                e = 1e-6 * A + 3e-7 * cap
                if wl.dtype == "f32":
                    tol = 2.0 ** -23 * np.abs(o) + (2e-5 + 2 * e) * w
                    ltol = 2e-5 + e + 2.0 ** -22 * np.abs(ref)
                else:
                    assert A <= 1000
                    tol = 2.0 ** -8 * np.abs(o) + (2.0 ** -8 + 1e-3) * w
                    ltol = 1e-3 + 2.0 ** -22 * np.abs(ref)
                err = np.abs(out[b, rows] - o)
                assert np.all(err <= tol), (what, l, b, h, float((err - tol).max()))
                assert np.all(np.abs(lse[b, rows] - ref) <= ltol), (what, l, b, h)
                worst = max(worst, float((err / tol).max()))
    say(f"{what}: {worst:.2f} of the tolerance")


DECODE = [  # dtype, d, gqa, H, Hp, B, ctx, cap, q_scale
    ("bf16", 128, 4, 4, 2, 3, (40, 900), 50.0, 3.0), ("bf16", 128, 16, 2, 2, 2, (100, 1500), 2.0, 3.0),
    ("bf16", 64, 8, 2, 1, 3, (40, 900), 30.0, 4.0), ("bf16", 64, 1, 4, 2, 5, (1, 300), 5.0, 2.0),
    ("bf16", 64, 4, 4, 2, 2, (200, 600), 5.0, 2.0), ("bf16", 64, 3, 4, 2, 2, (200, 600), 5.0, 2.0),
    ("bf16", 64, 2, 4, 2, 2, (200, 600), 5.0, 2.0), ("bf16", 64, 16, 1, 1, 1, 3000, 20.0, 4.0),
    ("f32", 64, 2, 4, 2, 2, 512, 50.0, 3.0), ("f32", 128, 1, 4, 2, 3, (1, 500), 2.0, 3.0),
    ("f32", 128, 3, 2, 2, 2, (20, 700), 30.0, 8.0), ("f32", 64, 1, 2, 2, 3, (20, 700), 0.001, 1.0),
    ("f32", 64, 3, 2, 2, 3, (20, 700), 1000.0, 1.0), ("f32", 128, 2, 2, 2, 3, (20, 700), 10.0, 1.0),
    ("f32", 64, 8, 2, 2, 2, (300, 900), 10.0, 4.0), ("f32", 128, 5, 4, 4, 2, (300, 900), 50.0, 4.0)]


@pytest.mark.parametrize("dtype,d,gqa,H,Hp,B,ctx,cap,q_scale", DECODE)
@pytest.mark.parametrize("n_bins,fused", [(4, False), (700, False), (40, True)])
def test_decode_capped(dtype, d, gqa, H, Hp, B, ctx, cap, q_scale, n_bins, fused):
    """Whole and split units, both merges, every kernel that a shape and a number of bins pick."""
    _gpu()
    wl = custom(31 + d + gqa, Geometry(2, H, H * gqa, d, 16, Hp), B, dtype, ctx, q_scale=q_scale, kv_scale=0.7)
    t = Tables(wl)
    pool = torch.from_numpy(poisoned_host_pool(wl, t)).to({"f32": torch.float32, "bf16": torch.bfloat16}[dtype]).cuda()
    s = DecodeSession(wl, tables=t, mode=tg.TG_PLAN_AOT_FILL, n_bins=n_bins, fill="host", pool=pool, fused_merge=fused,
                      softcap=cap)
    s.run_step()
    torch.cuda.synchronize()
    check_decode(s, cap, f"decode {dtype} d{d} gqa{gqa} bins {n_bins}")


def test_decode_capped_with_the_append_inside():
    """The in-launch append under a cap is tg_append followed by the capped decode, bit for bit."""
    _gpu()
    for dtype, d, gqa in (("bf16", 128, 4), ("bf16", 64, 8), ("f32", 64, 2), ("f32", 128, 8), ("bf16", 64, 1)):
        wl = custom(55, Geometry(2, 4, 4 * gqa, d, 16, 2), 3, dtype, (30, 400), q_scale=3.0)
        t = Tables(wl, headroom=np.full(3, 8, np.int32))
        outs = []
        for fused in (False, True):
            s = DecodeSession(wl, tables=t, mode=tg.TG_PLAN_AOT_FILL, n_bins=64, fill="host", open_end=True, softcap=6.0)
            gen = torch.Generator(device="cuda").manual_seed(3)
            shape = (2, 3, 4, d)
            k, v = (torch.randn(shape, generator=gen, device="cuda").to(s.dtype) for _ in range(2))
            s.enable_append(k, v, fused=fused)
            for _ in range(3):
                s.run_decode_step()
            torch.cuda.synchronize()
            outs.append((s.out, s.lse, s.live_len, s.pool))
            check_decode(s, 6.0, f"append {dtype} d{d} fused {fused}")
        assert all(torch.equal(a, b) for a, b in zip(*outs)), (dtype, d)


def test_decode_infinite_scores_are_capped():
    """+-infinite scores become +-softcap; a NaN score makes its head's output NaN and no other."""
    _gpu()
    for dtype, d, gqa in (("f32", 64, 2), ("bf16", 128, 4), ("f32", 128, 8), ("bf16", 64, 8)):
        wl = custom(56, Geometry(1, 2, 2 * gqa, d, 16, 1), 1, dtype, 100, ratio=np.ones((1, 1, 2)), q_scale=1.0)
        s = DecodeSession(wl, mode=tg.TG_PLAN_AOT_FILL, n_bins=8, fill="host", softcap=4.0)
        s.q[0, 0, 0] = 0
        s.q[0, 0, 0, 0] = 1.0            # head 0's scores are its keys' first dim
        page = int(s.t.pt_pages[int(s.t.pt_offsets[int(s.t.group_of[0, 0])])])
        s.pool[page, 0, 0, 1, 0], s.pool[page, 0, 0, 2, 0] = float("inf"), -float("inf")
        s.pool[page, 0, 0, 1, 1:], s.pool[page, 0, 0, 2, 1:] = 0, 0
        s.run_step()
        torch.cuda.synchronize()
        k, v = host_rows(f64(s.pool), s.t, wl.geom, 0, 0, 0, 100)
        z = 4.0 * np.tanh(k[:, 0] / math.sqrt(d) / 4.0)
        p = np.exp(z - z.max())
        o, w = p @ v / p.sum(), p @ np.abs(v) / p.sum()
        got = f64(s.out[0, 0, 0])
        tol = 2.0 ** -7 * w + 1e-3 * w if dtype == "bf16" else 3e-5 * w
        assert np.all(np.abs(got - o) <= tol), (dtype, d)
        assert bool(torch.isfinite(s.out[0, 0, gqa:].float()).all())
