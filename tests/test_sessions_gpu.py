"""Sessions whose steps come now as rotated keys, now as projection rows."""
import numpy as np
import pytest
import torch

from workloads import Geometry, custom

pytestmark = pytest.mark.gpu

if torch.cuda.is_available():
    from paper_2606_06302_amd import tangram as tg
    from paper_2606_06302_amd.runner import DecodeSession, Tables


@pytest.mark.parametrize("fused", [False, True])
def test_steps_that_append_and_steps_that_project_alternate(fused):
    """Whichever was enabled first, and when nothing else was: the same cache, lengths and outputs."""
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    B, g, d = 3, Geometry(2, 4, 16, 128, 16, 2), 128
    wl = custom(72, g, B, "bf16", (30, 400))
    t = Tables(wl, headroom=np.full(B, 16, np.int32))
    gen = torch.Generator(device="cuda").manual_seed(4)
    randn = lambda *s: torch.randn(*s, generator=gen, device="cuda").bfloat16()
    steps = 8
    k, v = randn(steps, 2, B, 4, d), randn(steps, 2, B, 4, d)
    rows = randn(steps, 2, B, (16 + 8) * d)
    turns = torch.from_numpy(tg.tg_rope_freqs(d, 10000.0)[0].view(np.int64)).cuda()
    w = (1 + 0.1 * randn(d)).bfloat16()
    spec = tg.make_rope_spec(tg.TG_ROPE_HALF, d, turns, 1.0, True, 1e-6, 0.0, w, w)
    results = []
    for order in ("append first", "projection first", "each before its step"):
        s = DecodeSession(wl, tables=t, mode=tg.TG_PLAN_AOT_FILL, n_bins=32, fill="host", open_end=True)
        kt, vt, rt = torch.zeros_like(k[0]), torch.zeros_like(v[0]), torch.zeros_like(rows[0])
        positions = torch.arange(B, dtype=torch.int32, device="cuda") * 1000
        append, project = (lambda: s.enable_append(kt, vt, fused=fused)), (lambda: s.enable_projection(spec, rt, positions))
        if order != "each before its step":
            first, second = (append, project) if order == "append first" else (project, append)
            first(), second()
        # memory that was let go is handed out again, and overwritten
        scratch = [torch.full((n,), 0x7fffffff, dtype=torch.int32, device="cuda") for n in (1, 8, 16, 64, 128, 256) * 8]
        outs = []
        for i in range(steps):
            s.q.copy_(0.1 * i + torch.linspace(-1, 1, s.q.numel(), device="cuda").view_as(s.q))
            if i % 2:
                kt.copy_(k[i]), vt.copy_(v[i])
                if order == "each before its step":
                    append()
                s.run_decode_step()
            else:
                rt.copy_(rows[i])
                if order == "each before its step":
                    project()
                s.run_projected_step()
            outs.append(s.out.clone())
        torch.cuda.synchronize()
        assert all(bool((x == 0x7fffffff).all()) for x in scratch)
        assert int(s.full) == 0 and torch.equal(s.live_len.cpu(), torch.from_numpy(t.kv_len) + steps)
        results.append((s.pool, *outs))
    for other in results[1:]:
        assert all(torch.equal(a, b) for a, b in zip(results[0], other))
