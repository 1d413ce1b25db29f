"""AddressSanitizer / UndefinedBehaviorSanitizer run of the host code behind
the clipping and 4-bit calls (CPU): argument checks, sizes, workspaces and
launch plans.  Built by hipcc with the sanitizers on the host pass only and
without the operators' kernels; GPU code is never built with a sanitizer.
"""
import glob
import os
import subprocess

import pytest

from test_sanitizers import CSRC, HIPCC, ROOT, _run


def test_operators_host_code_under_asan_and_ubsan(tmp_path):
    rts = glob.glob("/opt/rocm/llvm/lib/clang/*/lib/linux/libclang_rt.asan-x86_64.so")
    if not (os.path.exists(HIPCC) and rts):
        pytest.skip("hipcc or the clang sanitizer runtime not available")
    lib = str(tmp_path / "libags_san_operators.so")
    cmd = [HIPCC, "--offload-arch=gfx950", "-O1", "-g", "-std=c++17",
           "-fPIC", "-shared", "-shared-libasan",
           "-Xarch_host", "-fsanitize=address",
           "-Xarch_host", "-fsanitize=undefined",
           "-Xarch_host", "-fno-omit-frame-pointer",
           "-I", os.path.join(ROOT, "include"), "-I", CSRC,
           os.path.join(CSRC, "ags_api.hip"), os.path.join(CSRC, "ags_plan.cpp"),
           os.path.join(ROOT, "tests", "sanitizer_stubs.hip"), "-o", lib]
    subprocess.run(cmd, check=True, capture_output=True)
    code = ("import sys; sys.path.insert(0, 'tests')\n"
            "from paper_2603_18112_amd import ags\n"
            f"ags.load_library({lib!r})\n"
            "import pytest\n"
            "sys.exit(pytest.main(['-q', '-p', 'no:cacheprovider', 'tests/test_clip_abi.py', "
            "'tests/test_mx_abi.py']))")
    out = _run(code, {"LD_PRELOAD": sorted(rts)[-1]}, tmp_path)
    assert " passed" in out
