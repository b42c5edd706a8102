"""The host side of csrc/nm_step.hip (8-bit integer products, embedding, AdamW) under AddressSanitizer and UndefinedBehaviorSanitizer, CPU only: compiled for the host
and linked with stub launchers (tests/san_step_driver.cpp).  No GPU code is sanitized."""
import os
import shutil

import pytest

from test_sanitizers import ENV, ROOT, SAN, _run


def test_step_validation_under_asan_and_ubsan(tmp_path):
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    if not os.path.exists(hipcc) or shutil.which("g++") is None:
        pytest.skip("needs hipcc (host-only compile of the ABI layer) and g++")
    rocm = os.environ.get("ROCM_PATH", "/opt/rocm")
    obj, exe = str(tmp_path / "nm_step_san.o"), str(tmp_path / "san_step")
    host_san = []
    for f in ("-fsanitize=address", "-fsanitize=undefined", "-fno-sanitize-recover=all"):
        host_san += ["-Xarch_host", f]
    _run([hipcc, "--offload-arch=gfx950", "--offload-host-only", "-O1", "-g", "-std=c++17", "-fPIC", *host_san, "-c",
          os.path.join(ROOT, "paper_2203_10991_amd", "csrc", "nm_step.hip"), "-o", obj], cwd=str(tmp_path))
    _run(["g++", "-std=c++17", *SAN, "-D__HIP_PLATFORM_AMD__", f"-I{rocm}/include", f"-I{ROOT}/include",
          os.path.join(ROOT, "tests", "san_step_driver.cpp"), obj, "-o", exe, f"-L{rocm}/lib", "-lamdhip64", f"-Wl,-rpath,{rocm}/lib"])
    r = _run([exe], env=ENV, timeout=300)
    assert "step sanitizer driver ok" in r.stdout
