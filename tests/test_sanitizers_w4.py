"""CPU-only AddressSanitizer / UndefinedBehaviorSanitizer build of the host side of the 4-bit weights and the block
residual: the C ABI, the choice of kernels and the launchers, compiled for the host only, with stubs of the product
kernels' launchers and of the HIP runtime (tests/sanitize/w4_stubs.cpp), driven by tests/sanitize/w4_driver.cpp."""
import concurrent.futures as cf
import os
import re
import subprocess

import pytest

from test_sanitizers import CLANG, CLANGXX, CSRC, ENV, HIPCC, INCLUDE, SAN, _run


def test_w4_and_residual_hosts_under_asan_ubsan(tmp_path):
    if not (os.path.exists(HIPCC) and os.path.exists(CLANGXX)):
        pytest.skip("ROCm compilers not available")
    host = [HIPCC, "-x", "hip", "--offload-host-only", "-O1", "-g", "-std=c++17", "-Xarch_host",
            "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined", "-fno-omit-frame-pointer",
            "-I", INCLUDE, "-I", CSRC, "-I", SAN]
    sources = [os.path.join(CSRC, f"{n}.hip") for n in ("api_w4", "api_residual", "w4_linear", "w4_fold", "residual")]
    sources += [os.path.join(SAN, f"{n}.cpp") for n in ("w4_stubs", "w4_driver")]
    objs = [os.path.basename(s) + ".o" for s in sources]
    with cf.ThreadPoolExecutor(4) as ex:
        list(ex.map(lambda so: _run([*host, "-c", so[0], "-o", so[1]], str(tmp_path)), zip(sources, objs)))
    # The device-code image symbols the host objects refer to are named per build.
    nm = _run(["nm", "-u", *objs], str(tmp_path)).stdout
    fatbins = sorted(set(re.findall(r"__hip_fatbin_[0-9a-f]+", nm)))
    (tmp_path / "images.c").write_text("".join(f"char {f}[16];\n" for f in fatbins) + "extern int none;\n")
    _run([CLANG, "-O1", "-c", "images.c", "-o", "images.o"], str(tmp_path))
    _run([CLANGXX, "-fsanitize=address,undefined", *objs, "images.o", "-o", "driver"], str(tmp_path))
    r = subprocess.run([str(tmp_path / "driver")], capture_output=True, text=True, env=ENV)
    assert r.returncode == 0 and "clean" in r.stdout, r.stdout + r.stderr
