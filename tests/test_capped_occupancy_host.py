"""tg_decode_max_ctas counts the uncapped decode kernels' workgroups; a plan of that many bins also runs at once with a cap
(CPU only: the source is compiled, nothing runs)."""
import os
import re
import shutil
import subprocess

import pytest

from paper_2606_06302_amd import build


def test_capped_kernels_run_as_many_workgroups():
    if not (os.path.exists(build.HIPCC) or shutil.which(build.HIPCC)):
        pytest.skip("no HIP compiler")
    src = "tg_decode.hip"
    r = subprocess.run([build.HIPCC, *build.HIP_FLAGS, *build.HIP_EXTRA.get(src, []), "--cuda-device-only", "-S", "-o",
                        os.devnull, "-Rpass-analysis=kernel-resource-usage", os.path.join(build.CSRC, src)],
                       stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    assert r.returncode == 0, r.stdout[-2000:]
    waves = dict(zip(re.findall(r"Function Name: (\S+)", r.stdout),
                     map(int, re.findall(r"Occupancy \[waves/SIMD\]: (\d+)", r.stdout))))
    capped = {k: v for k, v in waves.items() if "Lb1EEE" in k and "decode" in k}      # the last template argument is kCap
    assert len(capped) == 16
    assert {k: v for k, v in capped.items() if waves[k.replace("Lb1EEE", "Lb0EEE")] != v} == {}
