"""The attention kernels find fragments by turning bits of LDS addresses, which needs tiles that start at multiples of a row, and read statistics 16 bytes at a time.  Where the compiler puts an
array follows from what the array's declaration asks for, so that is looked at here, in the compiler's own listing of the declarations.  (CPU only.)"""
import os
import re
import shutil
import subprocess

import pytest

from paper_2203_10991_amd import build

ROW = {1: 64, 2: 128, 3: 256, 4: 256}                                        # bytes of a row in LDS, by blocks of 32 elements
ARRAY = re.compile(r"^@_ZZN2nm4attn\d+(attention_\w*?kernel)ILi\dELi(\d)E\S*?E\d+(lds|v_lds|lse_of|delta_of) = .*addrspace\(3\) global (.*) undef,.*align (\d+)", re.M)


@pytest.mark.parametrize("source,kernels", [("attention", {"attention_kernel"}), ("attention_grad", {"attention_dq_kernel", "attention_dkdv_kernel"})])
def test_tiles_start_with_a_row(source, kernels, tmp_path):
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    if shutil.which(hipcc) is None:
        pytest.skip("needs hipcc")
    listing = str(tmp_path / "listing.ll")
    r = subprocess.run([hipcc, *build.HIPCC_FLAGS, "-Xclang", "-disable-llvm-passes", "--offload-device-only", "-emit-llvm", "-S", os.path.join(build.CSRC, source + ".hip"), "-o", listing],
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    with open(listing) as f:
        found = ARRAY.findall(f.read())
    assert {k for k, *_ in found} == kernels and {int(b) for _, b, *_ in found} == {1, 2, 3, 4}
    for kernel, blocks, name, kind, align in found:
        if kind == "[16 x i8]":                                              # (v in registers: no tile)
            continue
        need = ROW[int(blocks)] if name in ("lds", "v_lds") else 16
        assert int(align) >= need, f"{kernel} with {blocks} blocks: {name} on a boundary of {align} bytes, {need} needed"
