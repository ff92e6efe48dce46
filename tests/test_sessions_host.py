"""What a session's packed calls point at (CPU only: nothing is launched)."""
import numpy as np
import pytest
import torch

from paper_2606_06302_amd import tangram as tg
from paper_2606_06302_amd.runner import DecodeSession, Tables
from workloads import Geometry, custom


def session(fused=False, softcap=0.0):
    wl = custom(71, Geometry(2, 4, 8, 64, 16, 2), 3, "f32", (20, 60))
    t = Tables(wl, device="cpu", headroom=np.full(3, 4, np.int32))
    return DecodeSession(wl, tables=t, mode=tg.TG_PLAN_AOT_FILL, n_bins=8, fill="host", device="cpu", open_end=True,
                         fused_merge=fused, softcap=softcap)


def project(s):
    g = s.wl.geom
    rows = torch.zeros(g.num_layers, 3, (g.num_q_heads + 2 * g.num_kv_heads) * g.head_dim)
    s.enable_projection(tg.make_rope_spec(), rows, torch.zeros(3, dtype=torch.int32))


def check(s, append, projection):
    """Every packed pointer is a tensor's that the session holds."""
    shared = dict(pt_offsets=s.d_offsets, group_of=s.d_group_of, slot_of=s.d_slot_of, live_len=s.live_len, full=s.full,
                  kv_pool=s.pool, pt_pages=s.t.d_pt_pages)
    calls = [getattr(s, name) for name, on in (("append_args", append), ("rope_append_args", projection)) if on]
    for args in calls:
        for l in s.layers:
            for name, t in shared.items():
                assert getattr(args[l], name) == t.data_ptr(), name
    if append:
        for l in s.layers:
            assert s.append_args[l].k_tok == s.k_tok[l].data_ptr() and s.append_args[l].v_tok == s.v_tok[l].data_ptr()
        assert bool(s.append_decode_args) == s.fused_append
        for l, a in s.append_decode_args.items():
            assert a.append_full == s.full.data_ptr() and a.append_k == s.k_tok[l].data_ptr()
            assert a.append_v == s.v_tok[l].data_ptr()


@pytest.mark.parametrize("fused", [False, True])
@pytest.mark.parametrize("order", ["append", "projection", "append projection", "projection append",
                                   "append projection append", "projection append projection"])
def test_appends_and_projections_of_one_session_keep_their_tensors(order, fused):
    """Either call may come first, or again: the other's packed calls go on pointing at tensors that are held."""
    s = session()
    for what in order.split():
        s.enable_append(fused=fused) if what == "append" else project(s)
    assert int(s.full) == 0
    check(s, "append" in order, "projection" in order)
    s.set_bin_weights(np.arange(1, 9, dtype=np.int32))
    check(s, "append" in order, "projection" in order)


@pytest.mark.parametrize("first,second", [("append", "append"), ("append", "projection"), ("projection", "append")])
def test_enabling_again_takes_the_tables_as_they_are(first, second):
    s = session()
    enable = dict(append=s.enable_append, projection=lambda: project(s))
    enable[first]()
    held = s.d_offsets
    s.t.pt_offsets, s.t.group_of = s.t.pt_offsets + 7, s.t.group_of[:, ::-1].copy()
    enable[second]()
    assert s.d_offsets is held
    for d, a in ((s.d_offsets, s.t.pt_offsets), (s.d_group_of, s.t.group_of), (s.d_slot_of, s.t.slot_of)):
        assert np.array_equal(d.numpy(), a)
    check(s, "append" in (first, second), "projection" in (first, second))


def test_enabling_clears_the_flag():
    s = session()
    s.enable_append()
    s.full.fill_(1)
    project(s)
    assert int(s.full) == 0


@pytest.mark.parametrize("cap", [-1.0, float("nan"), float("inf"), 1e-5])
def test_a_cap_that_is_none_is_refused(cap):
    """Not taken for no cap at all (the library refuses it on the host: nothing is launched)."""
    s = session(softcap=cap)
    for call in (lambda: s.run_layer(0), s.run_step):
        with pytest.raises(tg.TangramError) as e:
            call()
        assert e.value.code == tg.TG_ERR_INVALID_ARG
