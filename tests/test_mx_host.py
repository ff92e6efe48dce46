"""The quantised cache's host side: sizes, and the refusals of its calls (CPU only: nothing reaches the GPU)."""
import ctypes as C

import numpy as np
import pytest

from oracle import mx
from paper_2606_06302_amd import tangram as tg

FAKE = 1 << 20                     # an aligned address that is never read: every call below is refused on the host
INVALID, UNSUPPORTED, SMALL = tg.TG_ERR_INVALID_ARG, tg.TG_ERR_UNSUPPORTED, tg.TG_ERR_BUFFER_TOO_SMALL
GOOD = tg.make_mx_format(tg.TG_MX_FP8, tg.TG_MX_FP4)


def geom(d=64, page=16, H=4, Hq=8, Hp=2, L=2):
    return tg.tg_geometry(L, H, Hq, d, page, Hp)


def append_args(**kw):
    a = dict(geom=geom(), batch=1, layer=0, dtype=tg.TG_BF16, k_tok=FAKE, v_tok=FAKE, kv_pool=FAKE, pt_pages=FAKE,
             pt_offsets=FAKE, group_of=FAKE, slot_of=FAKE, live_len=FAKE)
    return tg.tg_append_args(**{**a, **kw})


def compress_args(**kw):
    a = dict(geom=geom(), batch=1, chunk_len=4, dtype=tg.TG_BF16, k_new=FAKE, v_new=FAKE, scores=FAKE, kv_pool=FAKE,
             pt_pages=FAKE, items=FAKE, num_items=1, chunk_tokens=FAKE, keep_count=FAKE, kept=FAKE)
    return tg.tg_compress_args(**{**a, **kw})


def unpack_args(**kw):
    a = dict(geom=geom(), batch=1, layer=0, dtype=tg.TG_BF16, format=GOOD, mx_pool=FAKE, pt_pages=FAKE, pt_offsets=FAKE,
             group_of=FAKE, slot_of=FAKE, len=FAKE, kv_pool=FAKE)
    return tg.tg_unpack_mx_args(**{**a, **kw})


def decode_args(**kw):
    a = dict(geom=geom(), batch=1, dtype=tg.TG_BF16, q=FAKE, kv_pool=FAKE, pt_pages=FAKE, items=FAKE, bin_offsets=FAKE,
             n_bins=1, num_items=1, out=FAKE)
    return tg.tg_decode_args(**{**a, **kw})


CALLS = {"append": lambda f=GOOD, **kw: tg.tg_append_mx(append_args(**kw), f),
         "compress": lambda f=GOOD, **kw: tg.tg_compress_mx(compress_args(**kw), f),
         "unpack": lambda f=GOOD, **kw: tg.tg_unpack_mx(unpack_args(format=f, **kw)),
         "decode": lambda f=GOOD, **kw: tg.tg_decode_mx(decode_args(**kw), f)}


def refused(call, code):
    with pytest.raises(tg.TangramError) as e:
        call()
    assert e.value.code == code and tg.tg_last_error()


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("kb", [4, 8])
@pytest.mark.parametrize("vb", [4, 8])
def test_page_bytes(d, kb, vb):
    form = {4: tg.TG_MX_FP4, 8: tg.TG_MX_FP8}
    want = mx.slab_bytes(d, kb, vb)
    assert want == 16 * d * (kb + vb) // 8 + d
    assert tg.tg_mx_page_bytes(geom(d), tg.make_mx_format(form[kb], form[vb])) == 2 * want
    # every byte of a slab belongs to exactly one place
    p = mx.Places(d, kb, vb)
    seen = np.zeros(p.bytes, int)
    for bits, byte, bit, scale in p.parts:
        np.add.at(seen, byte.reshape(-1), bits)
        np.add.at(seen, scale.reshape(-1), 8)
    assert np.all(seen == 8)


def test_reference_rounding():
    """The reference itself, on values whose codes are known."""
    assert mx.magnitudes(4).tolist() == [0, 0.5, 1, 1.5, 2, 3, 4, 6] and mx.magnitudes(8)[-1] == 448 and mx.magnitudes(8)[1] == 2.0 ** -9
    row = np.zeros(32)
    row[:9] = [6.0, 5.0, 2.5, 0.25, 0.75, -0.25, -6.9, 3.5, 1.75]
    codes, scale = mx.quantise(row, 4)
    assert scale[0] == 127 and mx.values(codes, scale, 4)[:9].tolist() == [6, 4, 2, 0, 1, 0, -6, 4, 2]
    assert mx.quantise(np.full(32, 7.0), 4)[1][0] == 127 and mx.quantise(np.full(32, 7.01), 4)[1][0] == 128
    assert mx.quantise(np.full(32, 464.0), 8)[1][0] == 127 and mx.quantise(np.full(32, 464.1), 8)[1][0] == 128
    assert mx.quantise(np.r_[np.ones(31), np.nan], 8)[1][0] == 255 and np.isnan(mx.values(*mx.quantise(np.full(32, np.inf), 4), 4)).all()


@pytest.mark.parametrize("name", CALLS)
def test_formats_and_shapes(name):
    call = CALLS[name]
    for bad in (0, 5, 16, -4):
        refused(lambda: call(tg.make_mx_format(bad, tg.TG_MX_FP4)), INVALID)
        refused(lambda: call(tg.make_mx_format(tg.TG_MX_FP4, bad)), INVALID)
    for g, code in ((geom(96), UNSUPPORTED), (geom(256), UNSUPPORTED), (geom(page=32), UNSUPPORTED), (geom(Hp=3), INVALID),
                    (geom(H=0), INVALID)):
        refused(lambda: call(geom=g), code)
    refused(lambda: call(batch=0), INVALID)
    with pytest.raises(tg.TangramError):
        call(dtype=2)


@pytest.mark.parametrize("name,fields", [
    ("append", "k_tok v_tok kv_pool pt_pages pt_offsets group_of slot_of live_len"),
    ("compress", "k_new v_new scores kv_pool pt_pages items chunk_tokens keep_count kept"),
    ("unpack", "mx_pool pt_pages pt_offsets group_of slot_of len kv_pool"),
    ("decode", "q kv_pool pt_pages items bin_offsets out")])
def test_null_and_misaligned_pointers(name, fields):
    for f in fields.split():
        refused(lambda: CALLS[name](**{f: None}), INVALID)
    for f in {"append": "k_tok v_tok kv_pool", "compress": "k_new v_new kv_pool", "unpack": "mx_pool kv_pool",
              "decode": "q kv_pool out"}[name].split():
        refused(lambda: CALLS[name](**{f: FAKE + 8}), INVALID)


@pytest.mark.parametrize("name", ["append", "unpack"])
def test_layers(name):
    for layer in (-1, 2):
        refused(lambda: CALLS[name](layer=layer), INVALID)


def test_null_arguments():
    lib, fmt = tg._lib, C.byref(GOOD)
    for fn in (lib.tg_append_mx, lib.tg_compress_mx):
        assert fn(None, fmt, None) == INVALID
    assert lib.tg_decode_mx(None, fmt, 0.0, None) == INVALID and lib.tg_unpack_mx(None, None) == INVALID
    assert lib.tg_append_mx(C.byref(append_args()), None, None) == INVALID
    assert lib.tg_compress_mx(C.byref(compress_args()), None, None) == INVALID
    assert lib.tg_decode_mx(C.byref(decode_args()), None, 0.0, None) == INVALID
    assert lib.tg_mx_page_bytes(None, fmt) == 0 and lib.tg_mx_page_bytes(C.byref(geom()), None) == 0
    refused(lambda: tg.tg_mx_page_bytes(geom(80), GOOD), INVALID)


def test_decode_refusals():
    call = CALLS["decode"]
    for s in (-0.5, float("nan"), float("inf")):
        refused(lambda: call(sm_scale=s), INVALID)
    for cap in (-1.0, 1e-4, 1e7, float("nan"), float("inf")):
        refused(lambda: tg.tg_decode_mx(decode_args(), GOOD, cap), INVALID)
    refused(lambda: call(geom=geom(Hq=4 * 17)), UNSUPPORTED)
    refused(lambda: call(append_k=FAKE), INVALID)
    refused(lambda: call(append_k=FAKE, append_v=FAKE), INVALID)              # no live lengths
    refused(lambda: call(live_len=FAKE, layer=7), INVALID)
    refused(lambda: call(num_partials=3), INVALID)                             # no splits
    refused(lambda: call(num_partials=3, unit_splits=FAKE, unit_partial_base=FAKE), SMALL)
    refused(lambda: call(num_partials=3, unit_splits=FAKE, unit_partial_base=FAKE, workspace=FAKE + 8,
                         workspace_bytes=1 << 20), INVALID)
    refused(lambda: call(n_bins=0), INVALID)
    call(num_items=0)                                                          # nothing to do


def test_compress_refusals():
    call = CALLS["compress"]
    refused(lambda: call(chunk_len=0), INVALID)
    refused(lambda: call(chunk_len=tg.TG_COMPRESS_MAX_CHUNK + 1), INVALID)
    refused(lambda: call(num_items=-1), INVALID)
    call(num_items=0)


def test_bins_refusals():
    lens = np.ones((1, 2, 4), np.int32)
    refused(lambda: tg.tg_decode_mx_bins(geom(), tg.TG_BF16, GOOD, 0, 0, 0, lens), INVALID)
    refused(lambda: tg.tg_decode_mx_bins(geom(), tg.TG_BF16, GOOD, 0, 1, 2, lens), INVALID)
    refused(lambda: tg.tg_decode_mx_bins(geom(), tg.TG_BF16, GOOD, 0, 1, 0, 0 * lens), INVALID)
    refused(lambda: tg.tg_decode_mx_bins(geom(), 7, GOOD), INVALID)
    refused(lambda: tg.tg_decode_mx_bins(geom(96), tg.TG_BF16, GOOD), UNSUPPORTED)


def test_struct_layout_matches_the_header(tmp_path):
    import os
    import shutil
    import subprocess
    cc = shutil.which("gcc") or shutil.which("cc")
    if cc is None:
        pytest.skip("no host C compiler")
    lines = ['#include <stdio.h>', '#include <stddef.h>', '#include "tangram.h"', "int main(void) {"]
    structs = {"tg_unpack_mx_args": tg.tg_unpack_mx_args, "tg_mx_format": tg.tg_mx_format}
    for name, cls in structs.items():
        lines.append(f'printf("{name} %zu\\n", sizeof({name}));')
        lines += [f'printf("{name}.{f[0]} %zu\\n", offsetof({name}, {f[0]}));' for f in cls._fields_]
    lines += ['printf("fp4 %d\\nfp8 %d\\n", TG_MX_FP4, TG_MX_FP8);', "return 0; }"]
    src = tmp_path / "layout.c"
    src.write_text("\n".join(lines))
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    subprocess.run([cc, "-std=c99", f"-I{root}/include", str(src), "-o", str(tmp_path / "layout")], check=True)
    got = dict(x.split() for x in subprocess.run([str(tmp_path / "layout")], capture_output=True, text=True,
                                                 check=True).stdout.splitlines())
    for name, cls in structs.items():
        assert int(got[name]) == C.sizeof(cls)
        for f in cls._fields_:
            assert int(got[f"{name}.{f[0]}"]) == getattr(cls, f[0]).offset, (name, f[0])
    assert (int(got["fp4"]), int(got["fp8"])) == (tg.TG_MX_FP4, tg.TG_MX_FP8)
