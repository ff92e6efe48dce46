"""The calls around the cache together, as a served layer uses them: tables from the request lengths on the device,
projection rows normalised, rotated and attended chunk by chunk under a cap and a mask, compressed into the pages, then
decode steps that store their own token.  Every stage against a 64-bit form of its own inputs."""
import math

import numpy as np
import pytest
import torch

from gpu_helpers import say
from test_score_mod_gpu import attend, f64
from workloads import Geometry, custom

pytestmark = pytest.mark.gpu

if torch.cuda.is_available():
    from paper_2606_06302_amd import tangram as tg
    from paper_2606_06302_amd.device import to_device
    from paper_2606_06302_amd.runner import CompressSession, DecodeSession, DeviceTables, PrefillSession, Tables


def rotated(x, w, positions, theta, factor):
    """Norm and rotation by halves of x [..., heads, d] (64 bits), positions [...]."""
    y = x / np.sqrt((x * x).mean(-1, keepdims=True) + 1e-6) * w
    r = 2 * len(theta)
    ang = positions[..., None, None] * theta
    a, b, c, s = y[..., :r // 2], y[..., r // 2:r], np.cos(ang) * factor, np.sin(ang) * factor
    return np.concatenate([a * c - b * s, b * c + a * s, y[..., r:]], -1)


def close(got, want, room=0.0):
    """One rounding to bf16 (2^-8) of a value, and what its fp32 work may add."""
    return np.all(np.abs(got - want) <= 2.0 ** -8 * np.abs(want) + room)


@pytest.mark.parametrize("d,gqa,rot", [(128, 4, 128), (64, 5, 32)])
def test_from_lengths_and_projection_rows_to_decode_steps(d, gqa, rot):
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    H, Hp, B, C, cap, steps = 4, 2, 3, 48, 12.0, 4
    g = Geometry(1, H, H * gqa, d, 16, Hp)
    tokens = np.array([[48, 31, 48], [48, 0, 20]])            # valid tokens of the two chunks of every request
    ctx = tokens.sum(0).astype(np.int32)
    wl = custom(91 + d, g, B, "bf16", ctx, chunk_len=C)
    headroom = np.full(B, steps, np.int32)
    host = Tables(wl, headroom=headroom)
    # the tables on the device, from lengths that are there
    t = DeviceTables(g, to_device(ctx, "cuda"), to_device(wl.ratio, "cuda"), to_device(host.group_of, "cuda"),
                     to_device(host.slot_of, "cuda"), to_device(host.free_pages, "cuda"), host.pool_pages,
                     host.pages_needed, headroom=to_device(headroom, "cuda"))
    t.run()
    t.check()
    assert np.array_equal(t.d_kv_len.cpu().numpy(), host.kv_len)
    assert np.array_equal(t.d_offsets.cpu().numpy(), host.pt_offsets)
    assert np.array_equal(t.d_pt_pages.cpu().numpy(), host.pt_pages)
    pool = torch.full((host.pool_pages, 2, Hp, 16, d), float("nan"), dtype=torch.bfloat16, device="cuda")

    gen = torch.Generator(device="cuda").manual_seed(5)
    randn = lambda *s: torch.randn(*s, generator=gen, device="cuda")
    wq, wk = ((1 + 0.2 * randn(d)).bfloat16() for _ in range(2))
    turns, factor = tg.tg_rope_freqs(rot, 10000.0, tg.TG_ROPE_YARN, 4.0, 32, 1.0, 32.0)
    theta = turns.astype(np.float64) / 2.0 ** 64 * 2 * math.pi
    d_turns = torch.from_numpy(turns.view(np.int64)).cuda()
    spec = tg.make_rope_spec(tg.TG_ROPE_HALF, rot, d_turns, factor, True, 1e-6, 0.0, wq, wk)
    nq, nk = g.num_q_heads * d, H * d
    scale = 1 / math.sqrt(d)

    stored = np.zeros((B, 1, H), np.int32)                    # entries of every head so far
    start = np.zeros(B, np.int32)
    for chunk in range(2):
        n = tokens[chunk].astype(np.int32)
        d_n = to_device(n, "cuda")
        rows = (2 * randn(B * C, nq + 2 * nk)).bfloat16()
        q, k, v = (torch.zeros(B, C, heads, d, dtype=torch.bfloat16, device="cuda") for heads in (g.num_q_heads, H, H))
        tg.tg_rope(tg.make_rope_args(g, B, C, tg.TG_BF16, spec, rows[:, :nq], rows[:, nq:nq + nk], rows[:, nq + nk:], q, k, v,
                                     start=to_device(start, "cuda"), chunk_tokens=d_n))
        # attention over the compressed history and the chunk: the first quarter of it is seen by all of it
        at = np.tile(np.arange(C, dtype=np.int32), (B, 1))
        end = to_device(np.maximum(at + 1, C // 4).astype(np.int32), "cuda")
        mod = tg.make_score_mod(cap, d_n, None, end)
        s = PrefillSession(wl, tables=host, pool=pool, hist_len=stored, mod=mod)
        s.q.copy_(q), s.k_new.copy_(k), s.v_new.copy_(v)
        s.run()
        # the chunk's rows with the highest scores into the pages
        scores = randn(B, H, C)
        c = CompressSession(wl, host, pool, start, n, k_new=k, v_new=v, scores=scores)
        before = f64(pool)
        c.run()
        torch.cuda.synchronize()
        x = f64(rows).reshape(B, C, -1, d)
        pos = (start[:, None] + at).astype(np.float64)
        for b in range(B):
            i = slice(0, n[b])
            assert close(f64(q)[b, i], rotated(x[b, i, :g.num_q_heads], f64(wq), pos[b, i], theta, factor), 1e-4)
            assert close(f64(k)[b, i], rotated(x[b, i, g.num_q_heads:g.num_q_heads + H], f64(wk), pos[b, i], theta, factor), 1e-4)
            assert np.array_equal(f64(v)[b, i], x[b, i, g.num_q_heads + H:])
            for h in range(H):
                m = int(stored[b, 0, h])
                map_ = np.asarray([], np.int64)
                if m:
                    map_ = t.slot_map(0, m).cpu().numpy()[b, h]
                flat = before.reshape(-1, d)
                keys = np.concatenate([flat[map_], f64(k)[b, i, h]])
                vals = np.concatenate([flat[map_ + Hp * 16], f64(v)[b, i, h]])
                seen = np.ones((n[b], m + n[b]), bool)
                seen[:, m:] = at[b, None, i] < np.maximum(at[b, i] + 1, C // 4)[:, None]
                for j in range(h * gqa, (h + 1) * gqa):
                    o, w = attend(f64(q)[b, i, j], keys, vals, seen, scale, cap)
                    assert close(f64(s.out)[b, i, j], o, (2.0 ** -8 + 1e-3) * w), (chunk, b, j)
        # kept rows lie where the slot map says
        kept = c.kept.cpu().numpy()
        counts = c.plan["keep_count"]
        slots = t.slot_map(0, C, begin=to_device(stored, "cuda")).cpu().numpy()
        flat = f64(pool).reshape(-1, d)
        for b in range(B):
            for h in range(H):
                m = counts[b, h]
                assert np.array_equal(flat[slots[b, h, :m]], f64(k)[b, kept[b, h, :m], h])
                assert np.array_equal(flat[slots[b, h, :m] + Hp * 16], f64(v)[b, kept[b, h, :m], h])
        stored = stored + counts[:, None, :].astype(np.int32)
        start = start + n
    assert np.array_equal(stored, host.kv_len)

    # decode steps from projection rows, each captured token stored by the call itself
    ds = DecodeSession(wl, tables=host, mode=tg.TG_PLAN_AOT_FILL, n_bins=32, pool=pool, open_end=True, softcap=cap)
    positions = to_device(start, "cuda")
    rows = torch.zeros(1, B, nq + 2 * nk, dtype=torch.bfloat16, device="cuda")
    ds.enable_projection(spec, rows, positions)
    for step in range(steps + 1):
        rows.copy_((2 * randn(1, B, nq + 2 * nk)).bfloat16())
        ds.run_projected_step()
        torch.cuda.synchronize()
        full = step == steps                                   # the headroom is used up: nothing more is stored
        live = ds.live_len.cpu().numpy()
        longest = live.max()
        slots = t.slot_map(0, int(longest), length=ds.live_len).cpu().numpy()
        flat = f64(pool).reshape(-1, d)
        x = f64(rows[0]).reshape(B, -1, d)
        for b in range(B):
            qr = rotated(x[b, :g.num_q_heads], f64(wq), np.float64(start[b] + step), theta, factor)
            assert close(f64(ds.q[0])[b], qr, 1e-4)
            for h in range(H):
                m = int(live[b, 0, h])
                assert full or m == stored[b, 0, h] + step + 1
                at_ = slots[b, h, :m]
                assert (at_ >= 0).all() and (slots[b, h, m:] == -1).all()
                keys, vals = flat[at_], flat[at_ + Hp * 16]
                if m == stored[b, 0, h] + step + 1:
                    kr = rotated(x[b, g.num_q_heads + h:g.num_q_heads + h + 1], f64(wk), np.float64(start[b] + step), theta, factor)
                    assert close(keys[-1:], kr, 1e-4) and np.array_equal(vals[-1], x[b, g.num_q_heads + H + h])
                heads = slice(h * gqa, (h + 1) * gqa)
                o, w = attend(f64(ds.q[0])[b, heads], keys, vals, np.ones((gqa, m), bool), scale, cap)
                assert close(f64(ds.out[0])[b, heads], o, (2.0 ** -8 + 1e-3) * w), (step, b, h)
        positions.add_(1)
    say(f"d{d}: two chunks and {steps + 1} steps; {int(live.sum())} entries, full {int(ds.full)}")
