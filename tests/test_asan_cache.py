"""The cache's calls on the host under AddressSanitizer and UndefinedBehaviorSanitizer
(CPU only): api.hip (validation) and attend.hip (the split of the work) are compiled with
both on their host code, and tests/asan/cache_driver.c asks for splits over bounds from
nothing to the largest and calls the entry points with arguments that they refuse.
"""
import os
import shutil
import subprocess

import pytest

from tests.test_asan_host import CSRC, LLVM, ROOT, SANITIZE


def test_cache_calls_under_sanitizers(tmp_path):
    hipcc = shutil.which("hipcc") or "/opt/rocm/bin/hipcc"
    clang = os.path.join(LLVM, "clang")
    if not (os.path.exists(hipcc) and os.path.exists(clang)):
        pytest.skip("hipcc or ROCm's clang is not available")
    from paper_2609_13804_amd import binding
    lib_dir = os.path.dirname(binding.LIB_PATH)
    inc = ["-I", os.path.join(ROOT, "include"), "-I", CSRC]
    run = lambda cmd: subprocess.run(cmd, check=True, capture_output=True, text=True, timeout=600)
    objects = []
    for name in ("api", "attend"):
        objects.append(str(tmp_path / (name + ".o")))
        run([hipcc, "-O1", "-g", "-std=c++17", "-fPIC", "--offload-arch=gfx950", "-Xclang", "-target-feature",
             "-Xclang", "-packed-fp32-ops", *SANITIZE, *inc, "-c", os.path.join(CSRC, name + ".hip"),
             "-o", objects[-1]])
    driver, exe = str(tmp_path / "driver.o"), str(tmp_path / "driver")
    run([clang, "-std=c99", "-g", "-fsanitize=address,undefined", "-fno-sanitize-recover=all",
         "-D__HIP_PLATFORM_AMD__", *inc, "-I", "/opt/rocm/include", "-c",
         os.path.join(ROOT, "tests", "asan", "cache_driver.c"), "-o", driver])
    run([os.path.join(LLVM, "clang++"), "-fsanitize=address,undefined", driver, *objects,
         "-L", lib_dir, "-lstepprune", "-L", "/opt/rocm/lib", "-lamdhip64", "-lrocprofiler-sdk-roctx",
         f"-Wl,-rpath,{lib_dir}", "-Wl,-rpath,/opt/rocm/lib", "-o", exe])
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=0:abort_on_error=0",
               UBSAN_OPTIONS="print_stacktrace=1:halt_on_error=1")
    r = subprocess.run([exe], capture_output=True, text=True, timeout=120, env=env)
    assert r.returncode == 0, r.stdout + r.stderr
    assert r.stdout.strip().endswith("ok: 0 failure(s)"), r.stdout
