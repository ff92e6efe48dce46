"""Refusals of the attention calls with modified scores (CPU only: nothing reaches the GPU)."""
import ctypes as C

import pytest

from paper_2606_06302_amd import tangram as tg

G = tg.tg_geometry(2, 4, 8, 64, 16, 2)
FAKE = 1 << 20                     # an aligned address that is never read: every call below is refused on the host
INVALID, UNSUPPORTED = tg.TG_ERR_INVALID_ARG, tg.TG_ERR_UNSUPPORTED
BAD_CAPS = [-1.0, float("nan"), float("inf"), 1e-4, 1e7]


def prefill_args(**kw):
    a = dict(geom=G, batch=1, chunk_len=4, layer=0, dtype=tg.TG_BF16, q=FAKE, k_new=FAKE, v_new=FAKE, kv_pool=FAKE,
             pt_pages=FAKE, pt_offsets=FAKE, kv_len=FAKE, group_of=FAKE, slot_of=FAKE, out=FAKE)
    a.update(kw)
    return tg.tg_prefill_args(**a)


def decode_args(**kw):
    a = dict(geom=G, batch=1, dtype=tg.TG_BF16, q=FAKE, kv_pool=FAKE, pt_pages=FAKE, items=FAKE, bin_offsets=FAKE, n_bins=1,
             num_items=1, out=FAKE)
    a.update(kw)
    return tg.tg_decode_args(**a)


def refused(call, code):
    with pytest.raises(tg.TangramError) as e:
        call()
    assert e.value.code == code and tg.tg_last_error()


@pytest.mark.parametrize("cap", BAD_CAPS)
def test_caps_out_of_range(cap):
    refused(lambda: tg.tg_prefill_mod(prefill_args(), tg.make_score_mod(cap)), INVALID)
    refused(lambda: tg.tg_decode_capped(decode_args(), cap), INVALID)


def test_decode_needs_a_cap():
    refused(lambda: tg.tg_decode_capped(decode_args(), 0.0), INVALID)


@pytest.mark.parametrize("scale", [-0.1, float("nan"), float("inf")])
def test_scales(scale):
    refused(lambda: tg.tg_prefill_mod(prefill_args(sm_scale=scale), tg.make_score_mod(0.0)), INVALID)
    refused(lambda: tg.tg_prefill_mod(prefill_args(sm_scale=scale), tg.make_score_mod(5.0)), INVALID)
    refused(lambda: tg.tg_decode_capped(decode_args(sm_scale=scale), 5.0), INVALID)


def test_a_scale_that_the_cap_cannot_take():
    refused(lambda: tg.tg_prefill_mod(prefill_args(sm_scale=3e38), tg.make_score_mod(1e-3)), INVALID)
    refused(lambda: tg.tg_decode_capped(decode_args(sm_scale=3e38), 1e-3), INVALID)


@pytest.mark.parametrize("kw,code", [(dict(dtype=tg.TG_F32), UNSUPPORTED), (dict(chunk_len=0), INVALID),
                                     (dict(layer=2), INVALID), (dict(q=None), INVALID), (dict(out=FAKE + 8), INVALID),
                                     (dict(geom=tg.tg_geometry(2, 4, 8, 96, 16, 2)), UNSUPPORTED),
                                     (dict(geom=tg.tg_geometry(2, 4, 8, 64, 8, 2)), UNSUPPORTED),
                                     (dict(block_order=FAKE, num_blocks=0), INVALID)])
def test_prefill_refusals_are_those_of_tg_prefill(kw, code):
    refused(lambda: tg.tg_prefill_mod(prefill_args(**kw), tg.make_score_mod(5.0)), code)
    refused(lambda: tg.tg_prefill(prefill_args(**kw)), code)


@pytest.mark.parametrize("kw,code", [(dict(batch=0), INVALID), (dict(q=None), INVALID), (dict(q=FAKE + 8), INVALID),
                                     (dict(dtype=9), INVALID), (dict(append_k=FAKE), INVALID),
                                     (dict(num_partials=3), INVALID),
                                     (dict(geom=tg.tg_geometry(2, 1, 17, 64, 16, 1)), UNSUPPORTED)])
def test_decode_refusals_are_those_of_tg_decode(kw, code):
    refused(lambda: tg.tg_decode_capped(decode_args(**kw), 5.0), code)
    refused(lambda: tg.tg_decode(decode_args(**kw)), code)


def test_null_arguments():
    mod = tg.make_score_mod(5.0)
    assert tg._lib.tg_prefill_mod(None, C.byref(mod), None) == INVALID
    assert tg._lib.tg_prefill_mod(C.byref(prefill_args()), None, None) == INVALID
    assert tg._lib.tg_decode_capped(None, 5.0, None) == INVALID


def test_struct_layout_matches_the_header(tmp_path):
    import os
    import shutil
    import subprocess
    cc = shutil.which("gcc") or shutil.which("cc")
    if cc is None:
        pytest.skip("no host C compiler")
    s = tg.tg_score_mod
    lines = ['#include <stdio.h>', '#include <stddef.h>', '#include "tangram.h"', "int main(void) {",
             'printf("%zu\\n", sizeof(tg_score_mod));']
    lines += [f'printf("%zu\\n", offsetof(tg_score_mod, {f[0]}));' for f in s._fields_]
    (tmp_path / "l.c").write_text("\n".join(lines + ["return 0; }"]))
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    subprocess.run([cc, "-std=c99", f"-I{root}/include", str(tmp_path / "l.c"), "-o", str(tmp_path / "l")], check=True)
    got = [int(x) for x in subprocess.run([str(tmp_path / "l")], capture_output=True, text=True, check=True).stdout.split()]
    assert got == [C.sizeof(s)] + [getattr(s, f[0]).offset for f in s._fields_]
