"""No call of the sweep over the paged calls' sizes (sanitize/paged_driver.cpp), whose pointers are made up, reaches a
launch: the host code is linked with a runtime of a few functions that ends the process at the first one."""
import os
import re
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HIPCC = "/opt/rocm/bin/hipcc"

RUNTIME = r"""
#include <cstdio>
#include <cstdlib>
#include <hip/hip_runtime.h>
extern "C" {
hipError_t __hipPushCallConfiguration(dim3 grid, dim3 block, size_t, hipStream_t)
{
    std::printf("launch of %u x %u work-groups of %u\n", grid.x, grid.y, block.x);
    std::fflush(stdout);
    std::_Exit(3);
}
hipError_t __hipPopCallConfiguration(dim3*, dim3*, size_t*, hipStream_t*) { std::_Exit(4); }
hipError_t hipLaunchKernel(const void*, dim3, dim3, void**, size_t, hipStream_t) { std::_Exit(4); }
hipError_t hipMemcpyAsync(void*, const void*, size_t, hipMemcpyKind, hipStream_t) { std::_Exit(5); }
hipError_t hipStreamSynchronize(hipStream_t) { std::_Exit(5); }
hipError_t hipGetLastError() { std::_Exit(5); }
void** __hipRegisterFatBinary(const void*) { static void* none; return &none; }
void __hipUnregisterFatBinary(void**) {}
void __hipRegisterFunction(void**, const void*, char*, const char*, unsigned, void*, void*, void*, void*, int*) {}
"""


def _run(cmd, **kw):
    r = subprocess.run(cmd, capture_output=True, text=True, **kw)
    assert r.returncode == 0, " ".join(cmd) + "\n" + r.stdout[-2000:] + r.stderr[-2000:]
    return r.stdout


@pytest.mark.skipif(not os.path.exists(HIPCC), reason="hipcc not found")
def test_the_sweep_of_refusals_launches_nothing(tmp_path):
    csrc, inc = os.path.join(ROOT, "paper_2607_02963_amd", "csrc"), os.path.join(ROOT, "include")
    host = [HIPCC, "--offload-arch=gfx950", "--cuda-host-only", "-O1", "-std=c++17", "-Wno-unused-command-line-argument",
            "-I", inc, "-I", csrc, "-c"]
    objs = []
    for f in (os.path.join(csrc, "paged.hip"), os.path.join(csrc, "paged_mfma.hip"),
              os.path.join(ROOT, "tests", "sanitize", "paged_driver.cpp")):
        objs.append(str(tmp_path / (os.path.basename(f) + ".o")))
        _run([*host, f, "-o", objs[-1]])
    # the device code that is not there
    names = sorted(set(re.findall(r"U (__hip_fatbin\w*)", _run(["nm", "-u", *objs]))))
    stub = tmp_path / "runtime.hip"
    stub.write_text(RUNTIME + "".join(f"extern const char {n}[8]; const char {n}[8] = {{0}};\n" for n in names) + "}\n")
    objs.append(str(tmp_path / "runtime.o"))
    _run([*host, str(stub), "-o", objs[-1]])
    exe = str(tmp_path / "driver")
    _run(["/opt/rocm/llvm/bin/clang++", *objs, "-o", exe])  # without the HIP runtime
    r = subprocess.run([exe], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and "ok" in r.stdout, (r.returncode, r.stdout, r.stderr)
