"""AddressSanitizer and UndefinedBehaviorSanitizer builds of the cache operators' host
side (capi.hip; the kernels and their launchers are linked but never run), on the CPU."""
import os

import pytest

from test_sanitize import ENV, HERE, HIPCC, run


@pytest.mark.skipif(not os.path.exists(HIPCC), reason="no hipcc")
def test_cache_operators_host_checks_under_asan_and_ubsan(tmp_path):
    from paper_2508_02751_amd import build as B
    others = [os.path.join(B.BUILD, os.path.splitext(s)[0] + ".o") for s in B.SOURCES
              if s != "capi.hip"]
    if not all(os.path.exists(o) for o in others):
        B.build()
    san = ["-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined"]
    capi, drv, exe = (str(tmp_path / n) for n in ("capi_san.o", "driver.o", "driver"))
    run([HIPCC, f"--offload-arch={B.ARCH}", "-std=c++17", "-O1", "-g", "-fno-omit-frame-pointer",
         *san, "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
         "-I", B.INCLUDE, "-I", B.CSRC, "-c", os.path.join(B.CSRC, "capi.hip"), "-o", capi])
    run([HIPCC, "--offload-host-only", "-std=c++17", "-O1", "-g", *san, "-I", B.INCLUDE, "-c",
         "-x", "c++", os.path.join(HERE, "cache_abi_driver.cpp"), "-o", drv])
    run([HIPCC, f"--offload-arch={B.ARCH}", *san, drv, capi, *others, "-o", exe])
    r = run([exe], env=dict(ENV, ASAN_OPTIONS="detect_leaks=0"))
    assert "cache abi driver ok" in r.stdout
