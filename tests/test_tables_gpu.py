"""Block tables and slot maps built on the device: equal to the host's and the oracle's, bit for bit."""
import numpy as np
import pytest
import torch

import oracle
from gpu_helpers import say

pytestmark = pytest.mark.gpu

if torch.cuda.is_available():
    from paper_2606_06302_amd import tangram as tg


def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def cuda(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


class Admission:
    def __init__(self, B, L, H, Hp, P, ctx, ratio=None, budget=None, headroom=None, num_free=None, capacity=None, seed=0,
                 group_of=None, need=None):
        rng = np.random.default_rng(seed)
        self.geom = tg.tg_geometry(L, H, H, 64, P, Hp)
        self.B, self.L, self.H, self.G, self.P, self.Hp = B, L, H, H // Hp, P, Hp
        if ratio is None and budget is None:
            ratio = np.clip(rng.random((B, L, H)), 1e-3, 1.0)
            ratio[rng.random(ratio.shape) < 0.1] = 1.0
        self.ctx = np.array(np.broadcast_to(ctx, (B,)), np.int32)
        self.ratio, self.budget, self.headroom = ratio, budget, headroom
        if group_of is None:
            group_of = np.stack([rng.permutation(np.repeat(np.arange(self.G), Hp)) for _ in range(L)])
        self.group_of = np.asarray(group_of, np.int32)
        self.slot_of = np.zeros_like(self.group_of)
        for l in range(L):
            for g in range(self.G):
                at = self.group_of[l] == g
                self.slot_of[l, at] = np.arange(at.sum()) % Hp
        if need is None:
            need = tg.tg_reserve(self.geom, self.ctx, ratio, budget, self.group_of, np.zeros(0, np.int32), 0,
                                 size_query=True, headroom=headroom)["pages_needed"]
        self.need = need
        self.num_free = need + 7 if num_free is None else num_free
        self.capacity = need + 3 if capacity is None else capacity
        self.pool_pages = self.num_free + 11
        self.free = rng.permutation(self.pool_pages)[:self.num_free].astype(np.int32)

    def device(self, guard=64):
        """Outputs full of a pattern, the argument block; every output has a guard behind it."""
        n = self.B * self.L
        mark = -77
        o = dict(kv_len=torch.full((n * self.H + guard,), mark, dtype=torch.int32, device="cuda"),
                 group_len=torch.full((n * self.G + guard,), mark, dtype=torch.int32, device="cuda"),
                 offsets=torch.full((n * self.G + 1 + guard,), mark, dtype=torch.int64, device="cuda"),
                 pages=torch.full((self.capacity + guard,), mark, dtype=torch.int32, device="cuda"),
                 needed=torch.full((1,), mark, dtype=torch.int64, device="cuda"),
                 status=torch.full((1,), mark, dtype=torch.int32, device="cuda"))
        ws = torch.full((tg.tg_reserve_device_workspace_bytes(self.geom, self.B),), 0xAB, dtype=torch.uint8, device="cuda")
        self.keep = [cuda(self.ctx), None if self.ratio is None else cuda(self.ratio),
                     None if self.budget is None else cuda(self.budget), cuda(self.group_of),
                     cuda(self.free) if self.num_free else torch.zeros(0, dtype=torch.int32, device="cuda"), ws,
                     None if self.headroom is None else cuda(np.asarray(self.headroom, np.int32))]
        a = tg.make_reserve_device_args(self.geom, self.B, *self.keep[:5], self.pool_pages, o["kv_len"], o["group_len"],
                                        o["offsets"], o["pages"][:self.capacity], o["needed"], o["status"], ws,
                                        headroom=self.keep[6])
        return o, a

    def run(self, stream=None):
        o, a = self.device()
        tg.tg_reserve_device(a, stream)
        torch.cuda.synchronize()
        return {k: v.cpu().numpy() for k, v in o.items()}

    def check_ok(self, got):
        want = tg.tg_reserve(self.geom, self.ctx, self.ratio, self.budget, self.group_of, self.free, self.pool_pages,
                             headroom=self.headroom)
        n = self.B * self.L
        assert got["status"][0] == tg.TG_OK and got["needed"][0] == want["pages_needed"]
        for name, size in (("kv_len", n * self.H), ("group_len", n * self.G)):
            assert np.array_equal(got[name][:size], want[name].reshape(-1)), name
            assert np.all(got[name][size:] == -77), name
        assert np.array_equal(got["offsets"][:n * self.G + 1], want["pt_offsets"])
        assert np.all(got["offsets"][n * self.G + 1:] == -77)
        k = want["pages_needed"]
        assert np.array_equal(got["pages"][:k], want["pt_pages"]) and np.all(got["pages"][k:] == -77)
        return want

    def check_refused(self, got, code):
        n = self.B * self.L * self.G
        assert got["status"][0] == code
        assert not got["offsets"][:n + 1].any() and np.all(got["offsets"][n + 1:] == -77)
        assert np.all(got["pages"][self.capacity:] == -77)


SHAPES = [  # B, L, H, Hp, P, contexts
    (1, 1, 1, 1, 16, 1), (2, 1, 4, 2, 16, 512), (1, 64, 8, 2, 16, 40000), (7, 3, 6, 3, 1, 33), (64, 5, 8, 4, 16, 9000),
    (3, 257, 2, 2, 16, 100), (300, 2, 8, 8, 32, 2000), (5, 2, 40, 1, 16, 131072)]


@pytest.mark.parametrize("B,L,H,Hp,P,ctx", SHAPES)
@pytest.mark.parametrize("headroom", [False, True])
def test_tables_equal_the_hosts(B, L, H, Hp, P, ctx, headroom):
    _gpu()
    rng = np.random.default_rng(B + L)
    lens = rng.integers(max(1, ctx // 3), ctx, size=B, endpoint=True)
    a = Admission(B, L, H, Hp, P, lens, headroom=rng.integers(0, 50, B) if headroom else None, seed=B)
    got = a.run()
    want = a.check_ok(got)
    if not headroom and B * L * H < 4000:
        res = oracle.reserve(a.ratio, a.ctx, a.group_of, a.G, P, a.free)
        assert np.array_equal(got["kv_len"][:B * L * H].reshape(B, L, H), res["kv_len"])
        assert np.array_equal(got["offsets"][:B * L * a.G + 1], res["offsets"])
    say(f"tables B{B} L{L}: {want['pages_needed']} pages")


@pytest.mark.parametrize("num_free", [None, 20000])
@pytest.mark.parametrize("shift", [0, 1, 3])
def test_one_workgroup_and_many_page_lists_anywhere(num_free, shift):
    """The launch of small admissions and the two of large ones (a free list of 20000) give the same tables; page arrays
    need no more than their own alignment."""
    _gpu()
    for B, L, H, Hp, P in ((2, 1, 4, 2, 16), (16, 32, 8, 4, 16), (1, 1024, 1, 1, 16), (4, 64, 16, 4, 16)):
        a = Admission(B, L, H, Hp, P, np.arange(1, B + 1) * 37, headroom=np.full(B, 3, np.int32), seed=B)
        a = Admission(B, L, H, Hp, P, a.ctx, headroom=a.headroom, seed=B, num_free=num_free and max(num_free, a.need))
        o, args = a.device()
        free = torch.zeros(a.num_free + 4, dtype=torch.int32, device="cuda")
        free[shift:shift + a.num_free] = a.keep[4]
        pages = torch.full((a.capacity + 64,), -77, dtype=torch.int32, device="cuda")
        args.free_pages, args.pt_pages = free.data_ptr() + 4 * shift, pages.data_ptr() + 4 * shift
        tg.tg_reserve_device(args)
        torch.cuda.synchronize()
        assert bool((pages[:shift] == -77).all())
        o["pages"] = pages[shift:]
        a.check_ok({k: v.cpu().numpy() for k, v in o.items()})


def test_budget_instead_of_ratio_exact_products_and_one_long_request():
    _gpu()
    rng = np.random.default_rng(3)
    # ratios whose products with the length are whole numbers or a rounding away from one
    budget = np.array([[0.1, 0.3, 1 / 3, 0.7, 1.0, 2 ** -31, np.nextafter(0.5, 1), 0.5]])
    for ctx in (10, 30, 100, 2 ** 20, 2 ** 31 - 1):
        a = Admission(1, 1, 8, 2, 2 ** 20 if ctx > 2 ** 21 else 16, [ctx], budget=budget, seed=1)
        a.check_ok(a.run())
    a = Admission(4, 2, 4, 1, 16, rng.integers(1, 999, 4), budget=rng.random((2, 4)) * 0.9 + 0.05)
    a.check_ok(a.run())


def test_groups_of_unequal_size():
    """Any group ids in [0, G) are taken, as on the host: empty groups get empty tables."""
    _gpu()
    a = Admission(3, 2, 6, 2, 16, [100, 7, 4000], group_of=[[0, 0, 0, 0, 2, 2], [1, 1, 1, 1, 1, 1]])
    a.check_ok(a.run())


def test_exactly_enough_pages_and_capacity():
    _gpu()
    a = Admission(3, 2, 4, 2, 16, [100, 77, 4000])
    b = Admission(3, 2, 4, 2, 16, [100, 77, 4000], num_free=a.need, capacity=a.need)
    b.check_ok(b.run())


@pytest.mark.parametrize("what", ["pages", "capacity", "none"])
def test_too_few_pages(what):
    _gpu()
    full = Admission(3, 2, 4, 2, 16, [100, 77, 4000])
    kw = {"pages": dict(num_free=full.need - 1), "capacity": dict(capacity=full.need - 1),
          "none": dict(num_free=0, capacity=0)}[what]
    a = Admission(3, 2, 4, 2, 16, [100, 77, 4000], **kw)
    got = a.run()
    a.check_refused(got, tg.TG_ERR_BUFFER_TOO_SMALL if what == "capacity" else tg.TG_ERR_OUT_OF_PAGES)
    assert got["needed"][0] == full.need and np.all(got["pages"] == -77)


@pytest.mark.parametrize("B,L", [(3, 2), (70, 40)])
@pytest.mark.parametrize("bad", ["ctx", "ctx_negative", "ratio_zero", "ratio_nan", "ratio_big", "headroom", "group",
                                 "group_negative", "page_high", "page_negative"])
def test_invalid_inputs_leave_empty_tables(bad, B, L):
    _gpu()
    H, Hp = 4, 2
    a = Admission(B, L, H, Hp, 16, np.full(B, 300), headroom=np.zeros(B, np.int32), seed=4)
    if bad == "ctx":
        a.ctx[B - 1] = 0
    elif bad == "ctx_negative":
        a.ctx[0] = -5
    elif bad.startswith("ratio"):
        a.ratio[B // 2, L - 1, 3] = {"ratio_zero": 0.0, "ratio_nan": np.nan, "ratio_big": 1.0000001}[bad]
    elif bad == "headroom":
        a.headroom[1] = -1
    elif bad.startswith("group"):
        a.group_of[L - 1, 0] = 2 if bad == "group" else -1
    else:
        a.free[a.need - 1] = a.pool_pages if bad == "page_high" else -1
    got = a.run()
    a.check_refused(got, tg.TG_ERR_INVALID_ARG)


def test_a_bad_id_that_is_not_taken_does_no_harm():
    _gpu()
    a = Admission(3, 2, 4, 2, 16, [100, 77, 4000])
    a.free[a.need:] = -1
    got = a.run()
    assert got["status"][0] == tg.TG_OK
    a.free[a.need:] = np.setdiff1d(np.arange(a.pool_pages), a.free[:a.need])[:a.num_free - a.need]
    a.check_ok(got)


def slot_map(a, offsets, pages, layer, n, begin=None, length=None):
    out = torch.full((a.B * a.H * n + 32,), -77, dtype=torch.int64, device="cuda")
    keep = [cuda(offsets), cuda(pages), cuda(a.group_of), cuda(a.slot_of), None if begin is None else cuda(begin),
            None if length is None else cuda(length)]
    tg.tg_slot_map(tg.make_slot_map_args(a.geom, a.B, layer, *keep[:4], n, out, begin=keep[4], len=keep[5]))
    torch.cuda.synchronize()
    out = out.cpu().numpy()
    assert np.all(out[a.B * a.H * n:] == -77)
    return out[:a.B * a.H * n].reshape(a.B, a.H, n)


def plain_map(a, offsets, pages, layer, n, begin, length):
    out = np.full((a.B, a.H, n), -1, np.int64)
    for b in range(a.B):
        for h in range(a.H):
            t = (b * a.L + layer) * a.G + a.group_of[layer, h]
            cap = (offsets[t + 1] - offsets[t]) * a.P
            for j in range(n):
                e = j + (0 if begin is None else int(begin[b, layer, h]))
                if 0 <= e < cap and (length is None or e < length[b, layer, h]):
                    page = int(pages[offsets[t] + e // a.P])
                    out[b, h, j] = (page * 2 * a.Hp + int(a.slot_of[layer, h])) * a.P + e % a.P
    return out


@pytest.mark.parametrize("B,L,H,Hp,P,ctx,n", [(1, 1, 1, 1, 16, 1, 1), (2, 3, 4, 2, 16, 200, 17), (3, 2, 6, 3, 7, 90, 5),
                                              (2, 1, 4, 4, 16, 1500, 1300)])
def test_slot_maps(B, L, H, Hp, P, ctx, n):
    _gpu()
    a = Admission(B, L, H, Hp, P, np.full(B, ctx), headroom=np.full(B, 9, np.int32), seed=B)
    want = tg.tg_reserve(a.geom, a.ctx, a.ratio, None, a.group_of, a.free, a.pool_pages, headroom=a.headroom)
    kv = want["kv_len"]
    odd = kv.copy()
    odd.reshape(-1)[0] = -3          # a negative start: its first entries are none
    for layer in {0, L - 1}:
        for begin, length in ((None, None), (kv, None), (None, kv), (odd, None), (kv - 2, kv), (kv, np.zeros_like(kv))):
            got = slot_map(a, want["pt_offsets"], want["pt_pages"], layer, n, begin, length)
            ref = plain_map(a, want["pt_offsets"], want["pt_pages"], layer, n, begin, length)
            assert np.array_equal(got, ref), (layer, begin is None, length is None)


def test_slot_map_past_32_bits():
    """Page ids near the top of int32: rows past 2^31 (nothing is read at them)."""
    _gpu()
    a = Admission(1, 1, 4, 4, 16, [40], budget=np.ones((1, 4)))
    pages = np.array([2 ** 31 - 1, 2 ** 31 - 2, 5], np.int32)
    offsets = np.array([0, 3], np.int64)
    got = slot_map(a, offsets, pages, 0, 40)
    assert np.array_equal(got, plain_map(a, offsets, pages, 0, 40, None, None)) and got.max() > 2 ** 31


def test_two_streams_and_a_captured_graph():
    """Two admissions at once with workspaces of their own, and one captured: replays with new lengths equal the host."""
    _gpu()
    a, b = Admission(9, 30, 8, 2, 16, np.arange(1, 10) * 300, seed=1), Admission(5, 33, 4, 1, 16, np.arange(1, 6) * 77, seed=2)
    oa, aa = a.device()
    ob, ab = b.device()
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(3):
        tg.tg_reserve_device(aa, s1)
        tg.tg_reserve_device(ab, s2)
    torch.cuda.synchronize()
    a.check_ok({k: v.cpu().numpy() for k, v in oa.items()})
    b.check_ok({k: v.cpu().numpy() for k, v in ob.items()})
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s1):
        tg.tg_reserve_device(aa, s1)
    for i in range(4):
        a.ctx = (np.arange(9, 0, -1) * (100 + 50 * i)).astype(np.int32)      # no more pages than the list holds
        need = tg.tg_reserve(a.geom, a.ctx, a.ratio, None, a.group_of, a.free, a.pool_pages, size_query=True)["pages_needed"]
        assert need <= min(a.num_free, a.capacity)
        a.keep[0].copy_(cuda(a.ctx))
        oa["pages"].fill_(-77)
        graph.replay()
        torch.cuda.synchronize()
        a.check_ok({k: v.cpu().numpy() for k, v in oa.items()})
