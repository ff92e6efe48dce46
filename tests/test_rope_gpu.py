"""tg_rope and tg_rope_append against a plain 64-bit form.

Tolerance of a value that comes from the pair (a, b) after the norm, with f the factor of cosine and sine:
  2^-k |y| for the one rounding to the type (bf16: half a step, k = 8; f32: k = 24)
  + 2.5e-6 f (|a| + |b|) for the fp32 work, the sum of: the norm's sum of squares, at most 20 roundings in a row of
    2^-24 (1.2e-6 of the sum, 0.6e-6 of its root), its root and two products (3 more, 2e-7 with the root's own 1.2e-7),
    the angle (an eighth of a turn rounded to 24 bits, 2.4e-8, and 2^-32 of a turn dropped, 1.5e-9), the series (7
    roundings at most, 4.2e-7, the last ones dominating) and the rotation's products and sum (1.2e-7).
"""
import math

import numpy as np
import pytest
import torch

from gpu_helpers import say

pytestmark = pytest.mark.gpu

if torch.cuda.is_available():
    from paper_2606_06302_amd import tangram as tg

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
HALF_STEP = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}


def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def pairs(x, r, layout):
    """(members a, members b, rest) of the rotated pairs of x [..., d]."""
    if layout == "half":
        return x[..., :r // 2], x[..., r // 2:r], x[..., r:]
    return x[..., 0:r:2], x[..., 1:r:2], x[..., r:]


def join(a, b, rest, layout):
    head = np.concatenate([a, b], -1) if layout == "half" else np.stack([a, b], -1).reshape(*a.shape[:-1], -1)
    return np.concatenate([head, rest], -1)


def plain(x, positions, theta, r, layout, norm, w, eps, offset, factor):
    """(values, tolerance without the type's rounding) of x [tokens][heads][d] float64."""
    if norm:
        x = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * (1.0 if w is None else offset + w)
    a, b, rest = pairs(x, r, layout)
    # positions up to 2^31: the product in 64 bits of mantissa, whole turns dropped before it is rounded to 53
    ang = np.asarray(positions, np.longdouble)[:, None] * np.asarray(theta, np.longdouble)[None]
    two_pi = np.longdouble("6.283185307179586476925286766559")
    ang = (ang - np.floor(ang / two_pi) * two_pi).astype(np.float64)[:, None, :]
    c, s = np.cos(ang) * factor, np.sin(ang) * factor
    y = join(a * c - b * s, b * c + a * s, rest, layout)
    m = factor * (np.abs(a) + np.abs(b))
    return y, 2.5e-6 * join(m, m, np.abs(rest), layout)


class Case:
    def __init__(self, dtype, d, gqa, H, B, C, r, layout, norm, weights=True, offset=0.0, eps=1e-6, factor=1.0,
                 positions=None, scale=1.0, seed=0, pad=0):
        g = torch.Generator().manual_seed(seed)
        self.dtype, self.d, self.H, self.Hq, self.B, self.C, self.r = dtype, d, H, H * gqa, B, C, r
        self.layout, self.norm, self.offset, self.eps, self.factor = layout, norm, offset, eps, factor
        t = TYPES[dtype]
        heads = self.Hq + 2 * H
        rows = torch.randn(B * C, heads * d + pad, generator=g) * scale
        self.rows = rows.to(t).cuda()
        self.w = [(0.5 + torch.rand(d, generator=g)).to(t).cuda() if weights and norm else None for _ in range(2)]
        self.theta = 10000.0 ** (-2 * np.arange(max(1, r // 2)) / max(r, 1))
        self.turns = torch.from_numpy(tg.tg_rope_turns(self.theta).view(np.int64)).cuda()
        if positions is None:
            positions = torch.randint(0, 200000, (B, C), generator=g, dtype=torch.int32)
        self.positions = torch.as_tensor(np.asarray(positions), dtype=torch.int32).reshape(B, C).cuda()
        self.geom = tg.tg_geometry(1, H, self.Hq, d, 16, 1)
        self.tg_dtype = tg.TG_F32 if dtype == "f32" else tg.TG_BF16
        self.spec = tg.make_rope_spec(tg.TG_ROPE_HALF if layout == "half" else tg.TG_ROPE_INTERLEAVED, r, self.turns,
                                      factor, norm, eps, offset, self.w[0], self.w[1])

    def parts(self):
        q, k = self.Hq * self.d, self.H * self.d
        return self.rows[:, :q], self.rows[:, q:q + k], self.rows[:, q + k:q + 2 * k]

    def outputs(self):
        return [torch.full((self.B, self.C, n, self.d), float("nan"), dtype=TYPES[self.dtype], device="cuda")
                for n in (self.Hq, self.H, self.H)]

    def args(self, outs, **kw):
        return tg.make_rope_args(self.geom, self.B, self.C, self.tg_dtype, self.spec, *self.parts(), *outs,
                                 positions=kw.pop("positions", self.positions), **kw)

    def want(self, rows=None):
        """[(values, tolerance)] of q, k, v as [tokens][heads][d]."""
        res = []
        for i, x in enumerate(self.parts()):
            x = x.double().cpu().numpy().reshape(self.B * self.C, -1, self.d)
            if i == 2:
                res.append((x, np.zeros_like(x)))
                continue
            w = None if self.w[i] is None else self.w[i].double().cpu().numpy()
            y, tol = plain(x, self.positions.reshape(-1).cpu().numpy(), self.theta[:self.r // 2], self.r, self.layout,
                           self.norm, w, self.eps, self.offset, self.factor)
            res.append((y, tol + HALF_STEP[self.dtype] * np.abs(y)))
        return res

    def check(self, outs, what, valid=None):
        for name, o, (y, tol) in zip("qkv", outs, self.want()):
            got = o.double().cpu().numpy().reshape(y.shape)
            rows = np.ones(self.B * self.C, bool) if valid is None else valid.reshape(-1)
            err = np.abs(got[rows] - y[rows]) - tol[rows]
            assert np.all(np.isfinite(got[rows])), (what, name)
            assert err.max(initial=-1.0) <= 1e-30, (what, name, float(err.max()))
            assert np.all(np.isnan(got[~rows])), (what, name, "rows past the request's tokens were written")


SHAPES = [  # d, gqa, H, B, C, rot
    (128, 4, 8, 2, 5, 128), (128, 1, 1, 1, 1, 64), (64, 5, 8, 3, 33, 64), (64, 7, 2, 1, 2, 16), (128, 16, 2, 2, 3, 112),
    (64, 3, 3, 5, 7, 48), (128, 8, 8, 1, 1, 16), (64, 1, 4, 40, 1, 32), (128, 2, 4, 3, 4, 0)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("norm", [True, False])
@pytest.mark.parametrize("d,gqa,H,B,C,r", SHAPES)
def test_rope(dtype, layout, norm, d, gqa, H, B, C, r):
    _gpu()
    c = Case(dtype, d, gqa, H, B, C, r, layout, norm, seed=d + r + B)
    outs = c.outputs()
    tg.tg_rope(c.args(outs))
    torch.cuda.synchronize()
    c.check(outs, "rope")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_many_tokens_take_one_wave_each(dtype):
    """Enough tokens for the launch in which a wave walks all heads of its token, an odd head count among them."""
    _gpu()
    c = Case(dtype, 128, 3, 5, 9, 1001, 128, "half", True, seed=3)
    outs = c.outputs()
    tg.tg_rope(c.args(outs))
    torch.cuda.synchronize()
    c.check(outs, "rope many")


@pytest.mark.parametrize("positions", [0, 1, -1, 2 ** 31 - 1, -2 ** 31, 131072, 12345677])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_far_and_negative_positions(positions, layout):
    _gpu()
    c = Case("f32", 128, 2, 2, 1, 3, 128, layout, False, positions=np.full((1, 3), positions), seed=5)
    outs = c.outputs()
    tg.tg_rope(c.args(outs))
    torch.cuda.synchronize()
    c.check(outs, f"position {positions}")
    if positions == 0:      # nothing turns: bit for bit
        assert torch.equal(outs[0].reshape(3, -1), c.parts()[0]) and torch.equal(outs[2].reshape(3, -1), c.parts()[2])


@pytest.mark.parametrize("offset,eps,weights,factor,scale", [(1.0, 1e-6, True, 1.0, 1.0), (0.0, 0.0, True, 1.3, 1.0),
                                                             (1.0, 1e-5, False, 1.0, 1.0), (0.0, 1e-6, True, 1.0, 1e-6),
                                                             (0.0, 1e-6, True, 0.7, 1e6)])
def test_norm_variants(offset, eps, weights, factor, scale):
    _gpu()
    for dtype in ("bf16", "f32"):
        c = Case(dtype, 64, 2, 3, 2, 9, 32, "half", True, weights=weights, offset=offset, eps=eps, factor=factor,
                 scale=scale, seed=6)
        outs = c.outputs()
        tg.tg_rope(c.args(outs))
        torch.cuda.synchronize()
        c.check(outs, f"norm {offset} {eps} {weights} {factor} {scale}")


def test_a_row_of_zeros_stays_zero_and_values_pass_unchanged():
    _gpu()
    c = Case("bf16", 128, 2, 2, 1, 4, 128, "half", True, seed=7)
    q, k, v = c.parts()
    q[1], k[1] = 0, 0
    v[2] = float("inf")
    v[3, 5] = float("nan")
    outs = c.outputs()
    tg.tg_rope(c.args(outs))
    torch.cuda.synchronize()
    assert not outs[0][0, 1].any() and not outs[1][0, 1].any()
    assert torch.equal(outs[2].view(torch.int16).reshape(4, -1), v.contiguous().view(torch.int16))


@pytest.mark.parametrize("B,C,tokens", [(4, 13, [13, 0, 1, 7]), (2, 1, [0, 1]), (3, 700, [700, 699, 350])])
def test_requests_shorter_than_the_chunk(B, C, tokens):
    """Tokens past a request's length are not read (they hold NaN) and their outputs keep what they held."""
    _gpu()
    c = Case("bf16", 128, 4, 4, B, C, 128, "interleaved", True, seed=8)
    valid = np.arange(C)[None] < np.array(tokens)[:, None]
    c.rows.view(B, C, -1)[torch.from_numpy(~valid).cuda()] = float("nan")
    outs = c.outputs()
    tg.tg_rope(c.args(outs, chunk_tokens=torch.tensor(tokens, dtype=torch.int32, device="cuda")))
    torch.cuda.synchronize()
    c.check(outs, "ragged", valid)


def test_start_positions_equal_given_ones():
    _gpu()
    B, C = 3, 50
    start = torch.tensor([0, 99999, -20], dtype=torch.int32)
    c = Case("f32", 64, 2, 2, B, C, 64, "half", True, positions=start[:, None] + torch.arange(C, dtype=torch.int32), seed=9)
    a, b, z, zero = c.outputs(), c.outputs(), c.outputs(), c.outputs()
    tg.tg_rope(c.args(a))
    tg.tg_rope(c.args(b, positions=None, start=start.cuda()))
    tg.tg_rope(c.args(z, positions=None))
    at = torch.arange(C, dtype=torch.int32).expand(B, C).contiguous().cuda()
    tg.tg_rope(c.args(zero, positions=at))
    torch.cuda.synchronize()
    c.check(a, "positions")
    assert all(torch.equal(x, y) for x, y in zip(a, b)) and all(torch.equal(x, y) for x, y in zip(z, zero))


def test_parts_left_out_and_in_place():
    _gpu()
    c = Case("bf16", 128, 4, 2, 3, 11, 64, "half", True, seed=10, pad=64)    # rows wider than the heads
    outs = c.outputs()
    tg.tg_rope(c.args(outs))
    q, k, v = c.parts()
    for keep in ((0,), (1,), (2,), (0, 2), (1, 2), (0, 1)):
        ins = [x if i in keep else None for i, x in enumerate((q, k, v))]
        got = c.outputs()
        tg.tg_rope(tg.make_rope_args(c.geom, c.B, c.C, c.tg_dtype, c.spec, *ins,
                                     *[o if i in keep else None for i, o in enumerate(got)], positions=c.positions))
        torch.cuda.synchronize()
        for i in range(3):
            assert torch.equal(got[i], outs[i]) if i in keep else bool(torch.isnan(got[i]).all()), (keep, i)
    qd, kd, vd = (x.contiguous().clone() for x in (q, k, v))
    tg.tg_rope(tg.make_rope_args(c.geom, c.B, c.C, c.tg_dtype, c.spec, qd, kd, vd, qd, kd, vd, positions=c.positions))
    torch.cuda.synchronize()
    for o, x in zip(outs, (qd, kd, vd)):
        assert torch.equal(o.reshape(x.shape), x)


def test_stream_and_graph():
    """On a stream of its own, and captured: every replay equals the eager result for new inputs."""
    _gpu()
    c = Case("bf16", 128, 4, 8, 4, 65, 128, "half", True, seed=11)
    outs, want = c.outputs(), c.outputs()
    args, eager = c.args(outs), c.args(want)
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=st):
        tg.tg_rope(args, st)
    for i in range(4):
        c.rows.normal_()
        c.positions.add_(1000)
        tg.tg_rope(eager, torch.cuda.current_stream())
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(outs, want)), i


# ---------------------------------------------------------------- append
def tables(B, L, H, Hp, P, lens, cap_tokens, seed):
    """Page tables of cap_tokens entries per head and their placement."""
    rng = np.random.default_rng(seed)
    G = H // Hp
    group_of = np.stack([rng.permutation(np.repeat(np.arange(G), Hp)) for _ in range(L)]).astype(np.int32)
    slot_of = np.zeros_like(group_of)
    for l in range(L):
        for g in range(G):
            slot_of[l, group_of[l] == g] = np.arange(Hp)
    n = -(-cap_tokens // P)
    offsets = (np.arange(B * L * G + 1) * n).astype(np.int64)
    pages = rng.permutation(B * L * G * n + 5)[:B * L * G * n].astype(np.int32)
    c = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()
    live = torch.from_numpy(np.asarray(lens, np.int32).reshape(B, L, H)).cuda()
    return c(group_of), c(slot_of), c(offsets), c(pages), live, B * L * G * n + 5


@pytest.mark.parametrize("dtype,d,gqa,H,Hp,B,P,r,layout", [
    ("bf16", 128, 4, 8, 2, 1, 16, 128, "half"), ("bf16", 64, 5, 4, 4, 7, 16, 32, "interleaved"),
    ("f32", 64, 2, 4, 1, 33, 4, 64, "half"), ("f32", 128, 8, 2, 2, 3, 16, 48, "interleaved"),
    ("bf16", 128, 8, 8, 2, 64, 16, 128, "half"), ("bf16", 64, 1, 1, 1, 1, 1, 16, "half")])
def test_append_is_rope_then_append(dtype, d, gqa, H, Hp, B, P, r, layout):
    """Bit for bit what tg_rope and tg_append leave, in the pool, the lengths and the queries; heads whose table is
    full (or whose length is invalid) store nothing and raise the flag; other rows, layers and lengths stay."""
    _gpu()
    L, layer, cap = 3, 1, 3 * P
    rng = np.random.default_rng(B * d)
    lens = rng.integers(0, cap, (B, L, H))
    lens[0, layer, 0] = cap - 1
    if B > 2:
        lens[1, layer, H - 1], lens[2, layer, 0] = cap, -1
    c = Case(dtype, d, gqa, H, B, 1, r, layout, True, seed=B)
    c.geom = tg.tg_geometry(L, H, H * gqa, d, P, Hp)
    group_of, slot_of, offsets, pages, live, pool_pages = tables(B, L, H, Hp, P, lens, cap, B)
    pool = torch.randn(pool_pages, 2, Hp, P, d, device="cuda").to(TYPES[dtype])
    ref_pool, ref_live = pool.clone(), live.clone()
    q, k, v = c.outputs()
    full, ref_full = (torch.zeros(1, dtype=torch.int32, device="cuda") for _ in range(2))
    tg.tg_rope(c.args([q, k, v]))
    tg.tg_append(tg.make_append_args(c.geom, B, layer, c.tg_dtype, k, v, ref_pool, pages, offsets, group_of, slot_of,
                                     ref_live, ref_full))
    q2 = torch.full_like(q, float("nan"))
    tg.tg_rope_append(tg.make_rope_append_args(c.geom, B, layer, c.tg_dtype, c.spec, *c.parts(), c.positions, q2, pool,
                                               pages, offsets, group_of, slot_of, live, full))
    torch.cuda.synchronize()
    c.check([q, k, v], "rope")
    assert torch.equal(q, q2) and torch.equal(live, ref_live) and torch.equal(full, ref_full)
    assert torch.equal(pool, ref_pool)
    assert int(full) == (1 if B > 2 else 0)
    # without queries, without a flag
    again = live.clone()
    tg.tg_rope_append(tg.make_rope_append_args(c.geom, B, layer, c.tg_dtype, c.spec, None, *c.parts()[1:], c.positions,
                                               None, pool, pages, offsets, group_of, slot_of, again))
    torch.cuda.synchronize()
    grown = (live[:, layer] >= 0) & (live[:, layer] < cap)
    assert torch.equal(again[:, layer], live[:, layer] + grown.int())
    say(f"append {dtype} d{d} B{B}: {int(grown.sum())} heads stored")


def test_append_graph_replays():
    _gpu()
    B, H, Hp, P, d = 5, 4, 2, 16, 128
    c = Case("bf16", d, 4, H, B, 1, 128, "half", True, seed=21)
    c.geom = tg.tg_geometry(1, H, H * 4, d, P, Hp)
    group_of, slot_of, offsets, pages, live, pool_pages = tables(B, 1, H, Hp, P, np.full((B, 1, H), 3), 64, 2)
    pool = torch.zeros(pool_pages, 2, Hp, P, d, dtype=torch.bfloat16, device="cuda")
    ref_pool, ref_live = pool.clone(), live.clone()
    q, q2 = c.outputs()[0], c.outputs()[0]
    make = lambda q_, p_, l_: tg.make_rope_append_args(c.geom, B, 0, c.tg_dtype, c.spec, *c.parts(), c.positions, q_, p_,
                                                       pages, offsets, group_of, slot_of, l_)
    args, ref = make(q, pool, live), make(q2, ref_pool, ref_live)
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=st):
        tg.tg_rope_append(args, st)
    for i in range(5):
        c.rows.normal_()
        c.positions.add_(1)
        graph.replay()
        tg.tg_rope_append(ref, torch.cuda.current_stream())
        torch.cuda.synchronize()
        assert torch.equal(q, q2) and torch.equal(pool, ref_pool) and torch.equal(live, ref_live), i
    assert int(live.min()) == 8


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("f32", 64)])
def test_rows_and_pages_past_32_bits(dtype, d):
    """Projection rows whose second token lies past 2^32 bytes, and a pool whose pages do: bit for bit the result of
    dense ones."""
    _gpu()
    H, Hp, gqa, P = 4, 2, 2, 16
    c = Case(dtype, d, gqa, H, 2, 1, 32, "half", True, seed=31)
    c.geom = tg.tg_geometry(1, H, H * gqa, d, P, Hp)
    esz = c.rows.element_size()
    outs, far = c.outputs(), c.outputs()
    tg.tg_rope(c.args(outs))
    stride = (2 ** 32 + 2 ** 20) // esz
    wide = torch.empty(stride + c.rows.shape[1], dtype=c.rows.dtype, device="cuda")
    near = c.rows
    c.rows = torch.as_strided(wide, near.shape, (stride, 1))
    c.rows.copy_(near)
    tg.tg_rope(c.args(far))
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(outs, far))

    group_of, slot_of, offsets, pages, live, n = tables(2, 1, H, Hp, P, np.full((2, 1, H), 17), 48, 3)
    page = 2 * Hp * P * d
    shift = (2 ** 32 + 2 ** 20) // (page * esz)
    pools = [torch.zeros(n, 2, Hp, P, d, dtype=c.rows.dtype, device="cuda"),
             torch.empty(n + shift, 2, Hp, P, d, dtype=c.rows.dtype, device="cuda")]
    pools[1][shift:].zero_()
    q = [x[0] for x in (outs, far)]
    for pool, q_, pg, rows in zip(pools, q, (pages, pages + shift), (near, c.rows)):
        q_.fill_(float("nan"))
        c.rows = rows
        tg.tg_rope_append(tg.make_rope_append_args(c.geom, 2, 0, c.tg_dtype, c.spec, *c.parts(), c.positions, q_, pool, pg,
                                                   offsets, group_of, slot_of, live.clone()))
    torch.cuda.synchronize()
    assert torch.equal(*q) and torch.equal(pools[0], pools[1][shift:])
    assert int((pools[0] != 0).any(-1).sum()) == 2 * H * 2
