"""The host code of the 4-bit and cache entry points (argument checks, the attention's size
query) under AddressSanitizer and UndefinedBehaviorSanitizer, on the CPU: their sources built
with host-side instrumentation only, driven by a C++ program that enqueues nothing."""
import os
import subprocess

from test_host_asan import CSRC, ROOT, _hipcc
from paper_2609_07008_amd.build import SOURCES


def test_cache_host_code_under_sanitizers(tmp_path):
    cc = _hipcc()
    common = ["-O1", "-g", "-std=c++17", "-I" + os.path.join(ROOT, "include"), "-Wno-unused-command-line-argument",
              "-Xarch_host", "-fsanitize=address,undefined", "-Xarch_host", "-fno-sanitize-recover=undefined",
              "-Xarch_host", "-fno-omit-frame-pointer"]
    lib, drv = tmp_path / "libmla_asan.so", tmp_path / "driver"
    subprocess.run([cc, *common, "-fPIC", "-shared", "--offload-arch=gfx950", "-Xclang", "-target-feature", "-Xclang",
                    "-packed-fp32-ops", "-o", str(lib), *[os.path.join(CSRC, s) for s in SOURCES]], check=True, capture_output=True)
    subprocess.run([cc, *common, "-o", str(drv), os.path.join(ROOT, "tests", "host", "asan_cache_driver.cpp"), "-L" + str(tmp_path),
                    "-lmla_asan", "-Wl,-rpath," + str(tmp_path)], check=True, capture_output=True)
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=0:abort_on_error=1", UBSAN_OPTIONS="print_stacktrace=1:halt_on_error=1")
    r = subprocess.run([str(drv)], capture_output=True, text=True, timeout=600, env=env)
    assert r.returncode == 0, r.stdout[-2000:] + r.stderr[-4000:]
    assert "accepted without a row" in r.stdout
