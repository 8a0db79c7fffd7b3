"""The paged kernels are compiled with NaN semantics: hidden rows may hold NaNs, and a visible one is the result of the
rows that see it, so no operation may be taken to be free of them."""
import os
import subprocess

import pytest

from paper_2607_02963_amd import _build


@pytest.mark.skipif(not os.path.exists(_build.HIPCC), reason="hipcc not found")
@pytest.mark.parametrize("name", ["paged.hip", "paged_mfma.hip"])
def test_no_operation_is_taken_to_be_free_of_nans(name, tmp_path):
    out = str(tmp_path / "code.ll")
    subprocess.run([_build.HIPCC, *_build.HIP_FLAGS, *_build.SOURCE_FLAGS.get(name, []), "-I", _build.INCLUDE, "-I", _build.CSRC,
                    "--cuda-device-only", "-emit-llvm", "-S", "-Xclang", "-disable-llvm-passes",
                    os.path.join(_build.CSRC, name), "-o", out], check=True, capture_output=True)
    with open(out) as f:
        text = f.read()
    assert "paged_" in text and "fmul" in text
    assert " nnan " not in text and " fast " not in text and '"no-nans-fp-math"="true"' not in text
