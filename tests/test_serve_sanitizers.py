"""The host code of the long-context operators built with AddressSanitizer and
UndefinedBehaviorSanitizer (plain g++, CPU only): tests/sanitize/serve_driver.cpp
runs every entry point over small and extreme arguments with host stand-ins for
the launches and checks what each kernel would be given: grids, runs, and
partials and counters inside the workspace."""
import os
import shutil
import subprocess

import pytest

from test_sanitizers import ROOT, SAN, _run


@pytest.mark.skipif(shutil.which("g++") is None or not os.path.isdir("/opt/rocm/include"),
                    reason="needs g++ and the ROCm headers")
def test_host_code_of_the_long_context_operators(tmp_path):
    exe = str(tmp_path / "serve_driver")
    csrc = os.path.join(ROOT, "paper_2406_09297_amd", "csrc")
    here = os.path.join(ROOT, "tests", "sanitize")
    subprocess.check_call(["g++", "-std=c++17", *SAN, "-D__HIP_PLATFORM_AMD__",
                           "-I/opt/rocm/include", "-I", os.path.join(ROOT, "include"), "-I", csrc,
                           os.path.join(csrc, "mlkv.cpp"), os.path.join(csrc, "serve.cpp"),
                           os.path.join(here, "kernel_stubs.cpp"),
                           os.path.join(here, "serve_stubs.cpp"),
                           os.path.join(here, "serve_driver.cpp"),
                           "-L/opt/rocm/lib", "-lamdhip64", "-lrocblas",
                           "-Wl,-rpath,/opt/rocm/lib", "-o", exe], timeout=600)
    _run(exe)
