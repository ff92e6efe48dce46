"""Calls enqueued behind a reservation that the device refused find empty tables, also where a group id is out of range
and names none: nothing is stored, and no history is read."""
import numpy as np
import pytest
import torch

from gpu_helpers import say
from test_score_mod_gpu import Prefill, _gpu
from test_tables_gpu import Admission, cuda
from workloads import Geometry

pytestmark = pytest.mark.gpu

if torch.cuda.is_available():
    from paper_2606_06302_amd import tangram as tg

GROUPS = [2, -1, 2 ** 31 - 1, -2 ** 31]      # of tables with two groups a layer


@pytest.mark.parametrize("group", GROUPS)
@pytest.mark.parametrize("refused", [True, False])
def test_slot_maps_and_appends(group, refused):
    """Layer 0's head 1 has the bad id.  refused: the tables are the refused reservation's; else whole ones, of which the
    other heads' stay in use."""
    _gpu()
    B, L, H, Hp, P, d = 3, 2, 4, 2, 16, 64
    a = Admission(B, L, H, Hp, P, [100, 7, 300], headroom=np.full(B, 5, np.int32), seed=5)
    good = tg.tg_reserve(a.geom, a.ctx, a.ratio, None, a.group_of, a.free, a.pool_pages, headroom=a.headroom)
    a.group_of = a.group_of.copy()
    a.group_of[0, 1] = group
    o, args = a.device()
    tg.tg_reserve_device(args)
    offsets, pages, ids = o["offsets"], o["pages"], cuda(a.group_of)
    live = o["kv_len"][:B * L * H].clone().view(B, L, H)
    if not refused:
        offsets, pages, live = cuda(good["pt_offsets"]), cuda(good["pt_pages"]), cuda(good["kv_len"])
    pages = pages.clamp(min=0)                                   # whatever was there: ids of the pool
    slots = cuda(a.slot_of)
    n = 40
    out = torch.full((B, H, n), -77, dtype=torch.int64, device="cuda")
    tg.tg_slot_map(tg.make_slot_map_args(a.geom, B, 0, offsets, pages, ids, slots, n, out))
    gen = torch.Generator(device="cuda").manual_seed(1)
    rows = torch.randn(B, 3 * H * d, generator=gen, device="cuda")
    q, k, v = rows[:, :H * d], rows[:, H * d:2 * H * d], rows[:, 2 * H * d:]
    spec = tg.make_rope_spec()
    for rope in (True, False):
        pool = torch.zeros(a.pool_pages, 2, Hp, P, d, device="cuda")
        n_live, full = live.clone(), torch.zeros(1, dtype=torch.int32, device="cuda")
        q_out = torch.zeros(B, H, d, device="cuda")
        if rope:
            positions = torch.zeros(B, dtype=torch.int32, device="cuda")
            tg.tg_rope_append(tg.make_rope_append_args(a.geom, B, 0, tg.TG_F32, spec, q, k, v, positions, q_out, pool, pages,
                                                       offsets, ids, slots, n_live, full))
        else:
            kc, vc = k.contiguous(), v.contiguous()
            tg.tg_append(tg.make_append_args(a.geom, B, 0, tg.TG_F32, kc, vc, pool, pages, offsets, ids, slots, n_live, full))
        torch.cuda.synchronize()
        grown = (n_live - live).cpu().numpy()
        want = np.zeros((B, L, H), int)
        if not refused:
            want[:, 0, [0, 2, 3]] = 1
        assert np.array_equal(grown, want) and int(full) == 1
        assert int((pool != 0).any(-1).sum()) == 2 * want.sum()
        assert not rope or torch.equal(q_out.view(B, -1), q)
    if refused:
        assert o["status"].item() == tg.TG_ERR_INVALID_ARG and not offsets[:B * L * a.G + 1].any()
        assert bool((out == -1).all())
    else:
        assert bool((out[:, 1] == -1).all()) and bool((out[:, [0, 2, 3], 0] >= 0).all())


@pytest.mark.parametrize("group", GROUPS)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("split", [False, True])
def test_prefills_see_no_history(split, d, group):
    """One of four heads has the bad id, behind whole tables and behind the empty ones of a refused reservation: heads
    without a table attend to their chunk alone, the others to what they had."""
    _gpu()
    p = Prefill(41, 4, 2, d, 2, 2, 90, (200, 900), "causal", 0.0, split=split)
    g = Geometry(2, 4, 8, d, 16, 2)
    bad = p.t.group_of.copy()
    bad[1, 2] = group
    ids = cuda(bad)
    p.s.args.group_of = ids.data_ptr()
    empty = torch.zeros_like(p.s.d_offsets)
    hist = p.hist.copy()
    for offsets, none in ((p.s.d_offsets, [2]), (empty, range(g.num_kv_heads))):
        p.s.args.pt_offsets = offsets.data_ptr()
        p.hist = hist.copy()
        p.hist[:, 1, list(none)] = 0
        for call in ("mod", "plain"):
            p.s.out.fill_(float("nan"))
            if call == "mod":
                p.s.run()
            else:
                tg.tg_prefill(p.s.args)
            torch.cuda.synchronize()
            p.check(f"{call} group {group} split {split}")
    say("ok")
