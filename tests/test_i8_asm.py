"""The 8-bit integer product issues its LDS reads and MFMAs as asm statements: the check of test_lds_reads_in_flight on its compiled code (CPU only)."""
import os
import re
import shutil
import subprocess

import pytest

from paper_2203_10991_amd import build
from test_lds_reads_in_flight import _touched_too_early


@pytest.mark.parametrize("name", ["gemm_i8"])
def test_nothing_touches_a_register_before_its_asm_read_or_mfma_is_done(tmp_path, name):
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    if not os.path.exists(hipcc) and shutil.which(hipcc) is None:
        pytest.skip("needs hipcc")
    out = tmp_path / "a.s"
    r = subprocess.run([hipcc, *build.HIPCC_FLAGS, "-S", "--cuda-device-only", os.path.join(build.CSRC, f"{name}.hip"), "-o", str(out)], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    kernels, current = {}, None
    for number, line in enumerate(out.read_text().split("\n"), 1):
        start = re.match(r"(_Z\w+):", line)
        if start:
            current = kernels.setdefault(start.group(1), [])
        elif line.startswith(".Lfunc_end"):
            current = None
        elif current is not None:
            current.append((number, line))
    issued = [k for k, lines in kernels.items() if any("ds_read" in line for _, line in lines) and any("mfma" in line for _, line in lines)]
    assert issued
    for k in issued:
        found = _touched_too_early(kernels[k])
        assert not found, f"{k}: {len(found)} instructions, first {found[:4]}"
