"""Sessions whose steps come now as rotated keys, now as projection rows."""
import numpy as np
import pytest
import torch

from test_tables_gpu import Admission, cuda
from workloads import Geometry, custom

pytestmark = pytest.mark.gpu

if torch.cuda.is_available():
    from paper_2606_06302_amd import tangram as tg
    from paper_2606_06302_amd.runner import DecodeSession, DeviceTables, Tables


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


def device_tables(num_free=None):
    a = Admission(3, 2, 4, 2, 16, [100, 77, 4000], num_free=num_free)
    t = DeviceTables(a.geom, cuda(a.ctx), cuda(a.ratio), cuda(a.group_of), cuda(a.slot_of), cuda(a.free), a.pool_pages,
                     a.capacity)
    torch.cuda.synchronize()
    return a, t


@pytest.mark.parametrize("how", ["stream", "handle", "default behind another", "graph"])
def test_the_status_is_waited_for_wherever_the_tables_are_made(how):
    """Tables made on another stream than the current one, behind work that takes a while."""
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    full, _ = device_tables()
    for num_free in (None, full.need - 1):
        a, t = device_tables(num_free)
        with pytest.raises(AssertionError):
            t.check()
        side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
        if how == "graph":
            with torch.cuda.graph(graph, stream=torch.cuda.Stream()):
                t.run(torch.cuda.current_stream())
        on = torch.cuda.default_stream() if how == "default behind another" else side
        with torch.cuda.stream(on):
            torch.cuda._sleep(20_000_000)
            if how == "graph":
                graph.replay()
            else:
                t.run({"stream": side, "handle": side.cuda_stream}.get(how))
        with torch.cuda.stream(torch.cuda.Stream()):
            if num_free is None:
                t.check()
                assert int(t.d_needed) == a.need
            else:
                with pytest.raises(tg.TangramError) as e:
                    t.check()
                assert e.value.code == tg.TG_ERR_OUT_OF_PAGES


@pytest.mark.parametrize("handle", [False, True])
def test_a_slot_maps_memory_is_its_streams(handle):
    """The map is allocated for the stream that writes it: memory that work on the current stream still reads is not taken."""
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    a, t = device_tables()
    t.run()
    t.check()
    want = t.slot_map(1, 5000)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    busy = torch.full_like(want, 3)
    torch.cuda._sleep(20_000_000)
    sums = busy.sum()                  # enqueued, not run
    del busy
    got = t.slot_map(1, 5000, stream=side.cuda_stream if handle else side)
    torch.cuda.synchronize()
    assert int(sums) == 3 * want.numel() and torch.equal(got, want)
