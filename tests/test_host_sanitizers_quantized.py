"""The host code of the 8-bit projections and the 4-bit paged cache (argument checks, the products' plans, workspace sizes) under
AddressSanitizer and UndefinedBehaviorSanitizer, host side only, through calls that must be refused before anything is launched
(tests/host_sanitize_quantized.cpp).  No GPU is needed."""
import glob
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2408_08146_amd", "csrc")
OUT = os.path.join(ROOT, "_build", "host_sanitize_quantized")


def test_host_code_is_clean_under_asan_and_ubsan():
    hipcc = shutil.which("hipcc") or "/opt/rocm/bin/hipcc"
    if not os.path.exists(hipcc):
        pytest.skip("hipcc not available")
    sources = [os.path.join(CSRC, s) for s in ("koala_int8.hip", "koala_paged.hip")]
    driver = os.path.join(ROOT, "tests", "host_sanitize_quantized.cpp")
    deps = sources + [driver, *glob.glob(os.path.join(CSRC, "*.h")), *glob.glob(os.path.join(ROOT, "include", "*.h"))]
    if not os.path.exists(OUT) or os.path.getmtime(OUT) < max(os.path.getmtime(d) for d in deps):
        os.makedirs(os.path.dirname(OUT), exist_ok=True)
        cmd = [hipcc, "--offload-arch=gfx950", "-O1", "-g", "-std=c++17", "-Xarch_device", "-O3",
               "-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined",
               "-Xarch_host", "-fno-sanitize-recover=undefined",
               "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops", "-Wno-unused-command-line-argument",
               "-I", os.path.join(ROOT, "include"), "-I", CSRC, *sources, "-x", "hip", driver, "-o", OUT]
        res = subprocess.run(cmd, capture_output=True, text=True)
        assert res.returncode == 0, res.stderr[-3000:]
    assert b"__asan_init" in open(OUT, "rb").read()              # the sanitizer runtime is really linked in
    env = dict(os.environ, ASAN_OPTIONS="abort_on_error=0:detect_leaks=1", UBSAN_OPTIONS="print_stacktrace=1")
    res = subprocess.run([OUT], capture_output=True, text=True, env=env, timeout=120)
    assert res.returncode == 0, (res.stdout + res.stderr)[-3000:]
    assert "host sanitize quantized: ok" in res.stdout
