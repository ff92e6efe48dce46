"""A pool of the other kind, or too small a one, is refused before a kernel reads or writes past its end (CPU only: every
call is refused on the host)."""
import numpy as np
import pytest
import torch

from paper_2606_06302_amd import tangram as tg
from paper_2606_06302_amd.runner import CompressSession, DecodeSession, PrefillSession, Tables
from workloads import Geometry, custom

G = tg.tg_geometry(1, 2, 4, 64, 16, 2)
FMT = tg.make_mx_format(tg.TG_MX_FP8, tg.TG_MX_FP4)
ROWS = torch.zeros(3, 2, 2, 16, 64, dtype=torch.bfloat16)
BYTES = torch.zeros(3, tg.tg_mx_page_bytes(G, FMT), dtype=torch.uint8)


def tok(*shape):
    return torch.zeros(*shape, dtype=torch.bfloat16)


def i32(*shape):
    return torch.zeros(*shape, dtype=torch.int32)


def append(pool):
    return tg.make_append_args(G, 1, 0, tg.TG_BF16, tok(2, 64), tok(2, 64), pool, i32(3), i32(4), i32(2), i32(2), i32(2))


def compress(pool):
    return tg.make_compress_args(G, 1, 4, tg.TG_BF16, tok(4, 2, 64), tok(4, 2, 64), torch.zeros(2, 4), pool, i32(3), i32(9), 1,
                                 i32(1), i32(2), i32(2, 4))


def decode(pool):
    return tg.make_decode_args(G, 1, tg.TG_BF16, tok(4, 64), pool, i32(3), i32(9), i32(2), 1, 1, None, None, 0, tok(4, 64))


def prefill(pool):
    return tg.make_prefill_args(G, 1, 4, 0, tg.TG_BF16, tok(4, 4, 64), tok(4, 2, 64), tok(4, 2, 64), pool, i32(3), i32(4),
                                i32(2), i32(2), i32(2), tok(4, 4, 64))


CALLS = {"tg_append": (append, tg.tg_append, False), "tg_append_mx": (append, lambda a: tg.tg_append_mx(a, FMT), True),
         "tg_compress": (compress, tg.tg_compress, False),
         "tg_compress_mx": (compress, lambda a: tg.tg_compress_mx(a, FMT), True),
         "tg_decode": (decode, tg.tg_decode, False), "tg_decode_noalloc": (decode, tg.tg_decode_noalloc, False),
         "tg_decode_capped": (decode, lambda a: tg.tg_decode_capped(a, 1.0), False),
         "tg_decode_mx": (decode, lambda a: tg.tg_decode_mx(a, FMT), True), "tg_prefill": (prefill, tg.tg_prefill, False),
         "tg_prefill_mod": (prefill, lambda a: tg.tg_prefill_mod(a, tg.make_score_mod(1.0)), False)}


@pytest.mark.parametrize("name", CALLS)
def test_a_pool_of_the_other_kind_is_refused(name):
    if torch.cuda.is_available():
        pytest.skip("host tensors")
    pack, call, quantised = CALLS[name]
    with pytest.raises(tg.TangramError) as e:
        call(pack(ROWS if quantised else BYTES))
    assert e.value.code == tg.TG_ERR_INVALID_ARG and "kv_pool" in str(e.value)
    # its own kind passes these checks, as does a pointer that was put in later (no GPU here: the launch is what fails)
    for args in (pack(BYTES if quantised else ROWS), pack(ROWS if quantised else BYTES)):
        if args.kv_pool == (ROWS if quantised else BYTES).data_ptr():
            args.kv_pool = (BYTES if quantised else ROWS).data_ptr()
        with pytest.raises(tg.TangramError) as e:
            call(args)
        assert e.value.code == tg.TG_ERR_HIP


def test_the_read_probe_takes_rows():
    with pytest.raises(tg.TangramError) as e:
        tg.tg_read_probe(G, tg.TG_BF16, BYTES, i32(1), i32(1), 8, i32(8))
    assert e.value.code == tg.TG_ERR_INVALID_ARG


def workload(C=8):
    wl = custom(5, Geometry(2, 4, 8, 64, 16, 2), 2, "bf16", (30, 60), chunk_len=C)
    return wl, Tables(wl, device="cpu", headroom=np.full(2, 4, np.int32))


def sessions(wl, t):
    tokens = np.full(2, 8, np.int32)
    return {"decode": lambda pool: DecodeSession(wl, tables=t, n_bins=8, split_target=8, device="cpu", open_end=True, mx=FMT,
                                                 pool=pool, q=torch.zeros(2, 2, 8, 64, dtype=torch.bfloat16)),
            "prefill": lambda pool: PrefillSession(wl, tables=t, layer=1, device="cpu", fill="host", mx=FMT, mx_pool=pool),
            "compress": lambda pool: CompressSession(wl, t, pool, wl.ctx_len - tokens, tokens, device="cpu", mx=FMT,
                                                     k_new=tok(2, 8, 4, 64), v_new=tok(2, 8, 4, 64))}


@pytest.mark.parametrize("name", ["decode", "prefill", "compress"])
def test_sessions_check_a_quantised_pool(name):
    wl, t = workload()
    make, need = sessions(wl, t)[name], t.pool_pages * tg.tg_mx_page_bytes(wl.geom, FMT)
    make(torch.zeros(need, dtype=torch.uint8))
    make(torch.zeros(need + 5, dtype=torch.uint8))
    for bad in (torch.zeros(need - 1, dtype=torch.uint8), torch.zeros(need, dtype=torch.bfloat16),
                torch.zeros(t.pool_pages, 2, 2, 16, 64, dtype=torch.bfloat16), torch.zeros(need, 2, dtype=torch.uint8)[:, 0]):
        with pytest.raises(AssertionError):
            make(bad)


def test_a_session_of_rows_refuses_bytes():
    """The packed calls of a session carry the type of its pool, the copies with an append or stamps too."""
    wl, t = workload()
    need = t.pool_pages * tg.tg_mx_page_bytes(wl.geom, FMT)
    s = sessions(wl, t)["decode"](torch.zeros(need, dtype=torch.uint8))
    s.enable_append(fused=True)
    for args in (s.dplans[0].args, s.append_decode_args[1]):
        with pytest.raises(tg.TangramError) as e:
            tg.tg_decode(args)
        assert e.value.code == tg.TG_ERR_INVALID_ARG
    tokens = np.full(2, 8, np.int32)
    c = CompressSession(wl, t, torch.zeros(need, dtype=torch.uint8), wl.ctx_len - tokens, tokens, device="cpu",
                        k_new=tok(2, 8, 4, 64), v_new=tok(2, 8, 4, 64))
    with pytest.raises(tg.TangramError) as e:
        c.run()
    assert e.value.code == tg.TG_ERR_INVALID_ARG
