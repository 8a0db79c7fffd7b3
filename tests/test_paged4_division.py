"""The division of the 4-bit attention's work where units are weighed by their rows' tiles of 16 (csrc/paged_common.h), on
the CPU as in test_paged_division.py: every unit is taken once, a cut pair's work-groups follow each other, each with a
unit at least, and the notes name their states; lengths outside the contract stay inside the arrays."""
import os
import shutil
import subprocess

import pytest

import test_paged_division as plain


def weighed():
    main = plain.MAIN
    for a, b in (("paged_begin(a, w", "paged_begin<true>(a, w"), ("paged_next(a, run", "paged_next<true>(a, run"),
                 ("rows = 16 << in(0, 4)", "rows = 16 * in(1, 4)"), ("in(0, 6), in(1, 4)", "in(0, 18), in(6, 12)")):
        assert a in main
        main = main.replace(a, b)
    return main


@pytest.fixture(scope="module")
def program(tmp_path_factory):
    if shutil.which("g++") is None:
        pytest.skip("g++ not found")
    d = tmp_path_factory.mktemp("division4")
    shutil.copy(os.path.join(plain.CSRC, "paged_common.h"), d)
    (d / "pdec_common.h").write_text(plain.WAVE)
    (d / "main.cpp").write_text(weighed())
    exe = str(d / "division")
    subprocess.run(["g++", "-std=c++17", "-O1", "-g", "-fwrapv", "-Wno-attributes", str(d / "main.cpp"), "-o", exe], check=True)
    return exe


@pytest.mark.parametrize("what", ["batches", "junk"])
@pytest.mark.parametrize("seed", range(6))
def test_weighed_units(program, what, seed):
    plain._run(program, what, str(seed))
