"""The host code of the operators in 8 bits (validation, sizes, the choice of a way) under AddressSanitizer and UndefinedBehaviorSanitizer.

Their sources and the entry points' are compiled with the sanitizers on the host pass only and linked with tests/host_sanitize/block8_host_checks.cpp, which calls only what returns
before any GPU call; the launches of the other sources are left unresolved, as nothing reaches them.
"""
import os
import subprocess
from concurrent.futures import ThreadPoolExecutor

import pytest

from paper_2601_07396_amd import build as pkg_build
from test_host_sanitizers import CLANGXX, HOST_SAN, ROOT, _run


@pytest.mark.timeout(900)
def test_host_code_is_clean_under_asan_and_ubsan(tmp_path):
    if not os.path.exists(CLANGXX):
        pytest.skip("ROCm clang++ not found")
    flags = [f for f in pkg_build.HIPCC_FLAGS if f != "-O3"] + ["-O1"] + HOST_SAN
    csrc = os.path.join(ROOT, "paper_2601_07396_amd", "csrc")
    objs = {os.path.join(csrc, n + ".hip"): str(tmp_path / (n + ".o")) for n in ("svdcache_api", "rows8_kernels", "matmul8_kernels")}
    with ThreadPoolExecutor(max_workers=3) as pool:
        list(pool.map(lambda so: _run(["hipcc", *flags, "-c", "-o", so[1], so[0]]), objs.items()))
    drv, exe = str(tmp_path / "checks.o"), str(tmp_path / "checks")
    _run([CLANGXX, "-O1", "-g", "-std=c++17", "-fsanitize=address,undefined", "-fno-sanitize-recover=undefined", "-I", os.path.join(ROOT, "include"),
          "-c", "-o", drv, os.path.join(ROOT, "tests", "host_sanitize", "block8_host_checks.cpp")])
    _run([CLANGXX, "-fsanitize=address,undefined", "-Wl,--unresolved-symbols=ignore-in-object-files", "-o", exe, drv, *objs.values(),
          "-L/opt/rocm/lib", "-lamdhip64", "-Wl,-rpath,/opt/rocm/lib"])
    res = subprocess.run([exe], stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, timeout=300)
    assert res.returncode == 0, res.stdout[-4000:]
    assert "passed" in res.stdout and "runtime error" not in res.stdout and "AddressSanitizer" not in res.stdout
