"""The host logic of block tables, rotary positions and the append with them under AddressSanitizer and
UndefinedBehaviorSanitizer: a driver sweeps sizes, strides and specs, whose pointers are made up.  The host code is linked
with a runtime of a few functions that ends the process at the first launch, so that none of its calls is one."""
import os
import re
import subprocess

import pytest

from test_paged_refusals_launch_nothing import RUNTIME

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HIPCC = "/opt/rocm/bin/hipcc"


def _run(cmd, **kw):
    r = subprocess.run(cmd, capture_output=True, text=True, **kw)
    assert r.returncode == 0, " ".join(cmd) + "\n" + r.stdout[-3000:] + r.stderr[-3000:]
    return r.stdout


@pytest.mark.skipif(not os.path.exists(HIPCC), reason="hipcc not found")
def test_serving_host_logic_under_asan_and_ubsan(tmp_path):
    csrc, inc = os.path.join(ROOT, "paper_2607_02963_amd", "csrc"), os.path.join(ROOT, "include")
    san = ["-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined", "-Xarch_host",
           "-fno-sanitize-recover=undefined", "-Xarch_host", "-fno-omit-frame-pointer"]
    host = [HIPCC, "--offload-arch=gfx950", "--cuda-host-only", "-O1", "-g", "-std=c++17", "-Wno-unused-command-line-argument",
            "-I", inc, "-I", csrc]
    objs = []
    for f in (os.path.join(csrc, "paged.hip"), os.path.join(csrc, "paged_mfma.hip"), os.path.join(csrc, "paged_serving.hip"),
              os.path.join(ROOT, "tests", "sanitize", "serving_driver.cpp")):
        objs.append(str(tmp_path / (os.path.basename(f) + ".o")))
        _run([*host, *san, "-c", f, "-o", objs[-1]])
    names = sorted(set(re.findall(r"U (__hip_fatbin\w*)", _run(["nm", "-u", *objs]))))  # the device code that is not there
    stub = tmp_path / "runtime.hip"
    stub.write_text(RUNTIME + "".join(f"extern const char {n}[8]; const char {n}[8] = {{0}};\n" for n in names) + "}\n")
    objs.append(str(tmp_path / "runtime.o"))
    _run([*host, "-c", str(stub), "-o", objs[-1]])
    exe = str(tmp_path / "driver")
    _run(["/opt/rocm/llvm/bin/clang++", "-fsanitize=address,undefined", *objs, "-o", exe])  # without the HIP runtime
    env = dict(os.environ, UBSAN_OPTIONS="print_stacktrace=1", ASAN_OPTIONS="abort_on_error=1:detect_leaks=0")
    assert "ok" in _run([exe], env=env, timeout=300)
