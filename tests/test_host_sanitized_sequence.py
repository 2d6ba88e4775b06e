"""The host side of the sequence operators under AddressSanitizer + UndefinedBehaviorSanitizer, on the CPU.

As for the other entry points: the library's host code is built with the sanitizers (device code is compiled and never runs here), and a
small C++ driver walks the workspace queries and the argument checks, at the extremes of sizes and strides among others.
"""
import os
import subprocess
import sys
from concurrent.futures import ThreadPoolExecutor

import pytest
import torch

from test_host_sanitized import CLANGXX, CSRC, HIPCC, ROOT, SAN, SOURCES, _run

SEQUENCE = ["linear_attention.hip", "layer_norm.hip", "api_sequence.hip"]


@pytest.mark.skipif(not os.path.exists(HIPCC), reason="hipcc not installed")
@pytest.mark.skipif(torch.cuda.is_available(), reason="calls whose arguments are taken end at the launch only without a GPU")
def test_sequence_entry_points_under_address_and_ub_sanitizers(tmp_path):
    def compile_one(src):
        obj = str(tmp_path / src.replace(".hip", ".o"))
        _run([HIPCC, "--offload-arch=gfx950", "-O1", "-g", "-std=c++17", "-fPIC", "-Xclang", "-target-feature", "-Xclang",
              "-packed-fp32-ops", "-Xarch_device", "-O0"] + SAN + ["-c", os.path.join(CSRC, src), "-o", obj])
        return obj

    with ThreadPoolExecutor(max_workers=8) as ex:
        objs = list(ex.map(compile_one, SEQUENCE + SOURCES))
    lib = str(tmp_path / "librslx_san.so")
    _run([HIPCC, "--offload-arch=gfx950", "-shared", "-fPIC", "-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined", "-shared-libsan",
          "-o", lib] + objs)
    exe = str(tmp_path / "host_driver")
    _run([CLANGXX, "-std=c++17", "-g", "-O1", "-fsanitize=address", "-fsanitize=undefined", "-fno-sanitize-recover=undefined",
          "-shared-libsan", os.path.join(ROOT, "tests", "host_sanitize", "sequence_driver.cpp"), "-o", exe, lib, "-Wl,-rpath," + str(tmp_path)])
    env = dict(os.environ)
    rt = subprocess.run([CLANGXX, "-print-file-name=libclang_rt.asan-x86_64.so"], capture_output=True, text=True).stdout.strip()
    env["LD_LIBRARY_PATH"] = os.path.dirname(rt) + os.pathsep + env.get("LD_LIBRARY_PATH", "")
    # the HIP runtime keeps process-lifetime allocations: leak checking off; everything else at its default
    env["ASAN_OPTIONS"] = "detect_leaks=0:abort_on_error=0"
    env["UBSAN_OPTIONS"] = "print_stacktrace=1:halt_on_error=1"
    r = subprocess.run([exe], capture_output=True, text=True, env=env, timeout=300)
    sys.stdout.write(r.stdout[-3000:])
    assert r.returncode == 0, "%s\n%s" % (r.stdout[-4000:], r.stderr[-6000:])
    assert "all checks passed" in r.stdout
    assert "runtime error" not in r.stderr and "AddressSanitizer" not in r.stderr, r.stderr[-6000:]
