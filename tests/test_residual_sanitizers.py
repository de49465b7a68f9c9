"""The host side of the residual calls under AddressSanitizer and UndefinedBehaviorSanitizer (CPU only): its checks see the ends of every
argument's range, its launches are replaced by ones that do nothing."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
ENV = dict(os.environ, ASAN_OPTIONS="detect_leaks=1:abort_on_error=0:verify_asan_link_order=0", UBSAN_OPTIONS="halt_on_error=1:print_stacktrace=1")


@pytest.mark.skipif(shutil.which("hipcc") is None, reason="needs hipcc")
def test_residual_api_under_asan_and_ubsan(tmp_path):
    objs = []
    for src in (os.path.join(ROOT, "paper_2511_04214_amd", "csrc", "residual_api.hip"), os.path.join(ROOT, "tests", "sanitize", "residual_api_driver.cpp")):
        objs.append(str(tmp_path / (os.path.basename(src) + ".o")))
        cmd = ["hipcc", "--offload-arch=gfx950", "--offload-host-only", "-std=c++17", "-O1", "-g", "-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined",
               "-Xarch_host", "-fno-sanitize-recover=all", "-x", "hip", "-c", src, "-o", objs[-1]]
        r = subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
        assert r.returncode == 0, r.stdout[-3000:]
    exe = str(tmp_path / "driver")
    r = subprocess.run(["hipcc", "--offload-arch=gfx950", "-fsanitize=address,undefined", "-fno-gpu-sanitize", "-o", exe] + objs, stdout=subprocess.PIPE,
                       stderr=subprocess.STDOUT, text=True)
    assert r.returncode == 0, r.stdout[-3000:]
    r = subprocess.run([exe], env=ENV, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, timeout=300)
    assert r.returncode == 0 and "residual api sanitizer driver ok" in r.stdout, r.stdout[-3000:]
