"""The paged calls' host logic under AddressSanitizer and UndefinedBehaviorSanitizer: their two sources, instrumented
on the host side only, with a driver that sweeps sizes."""
import concurrent.futures
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HIPCC = "/opt/rocm/bin/hipcc"


def _run(cmd, **kw):
    r = subprocess.run(cmd, capture_output=True, text=True, **kw)
    assert r.returncode == 0, " ".join(cmd) + "\n" + r.stdout[-3000:] + r.stderr[-3000:]
    return r


@pytest.mark.skipif(not os.path.exists(HIPCC), reason="hipcc not found")
def test_paged_host_logic_under_asan_and_ubsan(tmp_path):
    csrc, inc = os.path.join(ROOT, "paper_2607_02963_amd", "csrc"), os.path.join(ROOT, "include")
    san = ["-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined", "-Xarch_host",
           "-fno-sanitize-recover=undefined", "-Xarch_host", "-fno-omit-frame-pointer"]
    flags = ["--offload-arch=gfx950", "-O1", "-g", "-std=c++17", "-fPIC", "-Xclang", "-target-feature", "-Xclang",
             "-packed-fp32-ops", "-Wno-unused-command-line-argument", "-I", inc, "-I", csrc]
    srcs = [os.path.join(csrc, "paged.hip"), os.path.join(csrc, "paged_mfma.hip"),
            os.path.join(ROOT, "tests", "sanitize", "paged_driver.cpp")]

    def compile_one(f):
        obj = str(tmp_path / (os.path.basename(f) + ".o"))
        _run([HIPCC, *flags, *san, "-c", f, "-o", obj])
        return obj

    with concurrent.futures.ThreadPoolExecutor(max_workers=3) as ex:
        objs = list(ex.map(compile_one, srcs))
    exe = str(tmp_path / "paged_driver")
    _run([HIPCC, "--offload-arch=gfx950", *san, *objs, "-o", exe])
    env = dict(os.environ, UBSAN_OPTIONS="print_stacktrace=1", ASAN_OPTIONS="abort_on_error=1:detect_leaks=0")
    assert "ok" in _run([exe], env=env, timeout=300).stdout
