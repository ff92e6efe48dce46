"""The binding takes pointers of tensors: one of another type, with strides or too short would be read as something else, or
past its end (CPU only: nothing is launched)."""
import pytest
import torch

from paper_2606_06302_amd import tangram as tg

B, L, H, C, d = 2, 2, 4, 3, 64
G = tg.tg_geometry(L, H, 8, d, 16, 2)
TABLES = B * L * 2


def i32(*shape):
    return torch.zeros(*shape, dtype=torch.int32)


def i64(*shape):
    return torch.zeros(*shape, dtype=torch.int64)


def f32(*shape):
    return torch.zeros(*shape)


def spec(**kw):
    a = dict(rot_dim=d, turns=i64(d // 2), norm=True, q_weight=f32(d), k_weight=f32(d))
    a.update(kw)
    return tg.make_rope_spec(**a)


def rope(spec_kw=None, **kw):
    n = B * C
    a = dict(q_in=f32(n, 8 * d), k_in=f32(n, H * d), v_in=f32(n, H * d), q_out=f32(n, 8, d), k_out=f32(n, H, d),
             v_out=f32(n, H, d), positions=i32(B, C), start=i32(B), chunk_tokens=i32(B))
    a.update(kw)
    return tg.make_rope_args(G, B, C, tg.TG_F32, spec(**(spec_kw or {})), **a)


def append(spec_kw=None, **kw):
    a = dict(q_in=f32(B, 8 * d), k_in=f32(B, H * d), v_in=f32(B, H * d), positions=i32(B), q_out=f32(B, 8, d),
             kv_pool=f32(5, 2, 2, 16, d), pt_pages=i32(5), pt_offsets=i64(TABLES + 1), group_of=i32(L, H), slot_of=i32(L, H),
             live_len=i32(B, L, H), full=i32(1))
    a.update(kw)
    return tg.make_rope_append_args(G, B, 0, tg.TG_F32, spec(**(spec_kw or {})), **a)


def reserve(**kw):
    a = dict(ctx_len=i32(B), ratio=torch.zeros(B, L, H, dtype=torch.float64), budget=torch.zeros(L, H, dtype=torch.float64),
             group_of=i32(L, H), free_pages=i32(9), pool_pages=9, kv_len=i32(B, L, H), group_len=i32(TABLES),
             pt_offsets=i64(TABLES + 1), pt_pages=i32(5), pages_needed=i64(1), status=i32(1),
             workspace=torch.zeros(64, dtype=torch.uint8), headroom=i32(B))
    a.update(kw)
    return tg.make_reserve_device_args(G, B, **a)


def slot_map(**kw):
    a = dict(pt_offsets=i64(TABLES + 1), pt_pages=i32(5), group_of=i32(L, H), slot_of=i32(L, H), n=7, map=i64(B, H, 7),
             begin=i32(B, L, H), len=i32(B, L, H))
    a.update(kw)
    return tg.make_slot_map_args(G, B, 0, **a)


def mod(**kw):
    a = dict(softcap=1.0, chunk_tokens=i32(B), key_begin=i32(B, C), key_end=i32(B, C))
    a.update(kw)
    return tg.make_score_mod(**a)


def test_right_ones_are_taken():
    assert rope().q_stride == 8 * d and append().k_stride == H * d and reserve().num_free == 9 and slot_map().n == 7
    assert mod().softcap == 1.0
    # larger ones, empty ones and none
    append(kv_pool=f32(50, 2, 2, 16, d), live_len=i32(100), full=None, q_in=None, q_out=None)
    reserve(free_pages=i32(0), ratio=None, headroom=None, kv_len=i32(1000))
    slot_map(begin=None, len=None), mod(chunk_tokens=None, key_begin=None, key_end=None)
    rope(dict(turns=torch.zeros(d // 2, dtype=torch.uint64)), v_in=None, v_out=None, positions=None, start=None)


def strided(t):
    return torch.stack([t, t], -1)[..., 0]


CALLS = [(rope, "q_in k_in v_in q_out k_out v_out positions start chunk_tokens"),
         (append, "q_in k_in v_in positions q_out kv_pool pt_pages pt_offsets group_of slot_of live_len full"),
         (reserve, "ctx_len ratio budget group_of free_pages kv_len group_len pt_offsets pt_pages pages_needed status headroom"),
         (slot_map, "pt_offsets pt_pages group_of slot_of map begin len"), (mod, "chunk_tokens key_begin key_end")]
OTHER = {torch.int32: torch.int64, torch.int64: torch.int32, torch.float64: torch.float32, torch.float32: torch.bfloat16}
SIZED = {"pt_pages", "free_pages", "kv_pool", "chunk_tokens", "key_begin", "key_end"}     # of any length, or of a call's


@pytest.mark.parametrize("call,name", [(c, n) for c, names in CALLS for n in names.split()])
def test_other_types_strides_and_sizes_are_refused(call, name):
    import inspect
    source = {}

    def capture(*a, **kw):
        source.update(kw)
        return original(*a, **kw)
    maker = {rope: "make_rope_args", append: "make_rope_append_args", reserve: "make_reserve_device_args",
             slot_map: "make_slot_map_args", mod: "make_score_mod"}[call]
    original = getattr(tg, maker)
    setattr(tg, maker, capture)
    try:
        call()
    finally:
        setattr(tg, maker, original)
    assert name in inspect.signature(original).parameters
    t = source[name]
    with pytest.raises(AssertionError):
        call(**{name: t.to(OTHER[t.dtype])})
    if t.numel() > 1:
        with pytest.raises(AssertionError):
            call(**{name: strided(t)})
    if name not in SIZED or call is rope:
        short = t[:-1] if t.dim() == 1 else t[:-1].contiguous()
        with pytest.raises(AssertionError):
            call(**{name: short})


@pytest.mark.parametrize("kw", [dict(q_weight=torch.zeros(d, dtype=torch.bfloat16)), dict(k_weight=strided(torch.zeros(d))),
                                dict(turns=torch.zeros(d // 2)), dict(turns=torch.zeros(d // 2 - 1, dtype=torch.int64))])
def test_weights_and_turns(kw):
    for call in (rope, append):
        with pytest.raises(AssertionError):
            call(kw)
