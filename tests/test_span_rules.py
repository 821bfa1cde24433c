"""The overlap check of the operators' entry points (host code, no GPU): compiled from the
library's internal header and compared with every byte of random layouts, and reached
through the entry points for column slices of one buffer."""

import os
import shutil
import subprocess

import pytest

from paper_1904_00962_amd import _lib, _ops, build

HERE = os.path.dirname(os.path.abspath(__file__))


def test_against_every_byte(tmp_path):
    gxx = shutil.which("g++")
    rocm = os.environ.get("ROCM_PATH", "/opt/rocm")
    if gxx is None or not os.path.exists(os.path.join(rocm, "include", "hip")):
        pytest.skip("needs g++ and the HIP headers")
    exe = tmp_path / "rules"
    r = subprocess.run([gxx, "-std=c++17", "-O2", "-D__HIP_PLATFORM_AMD__", "-I", build.INCLUDE,
                        "-I", build.CSRC, "-I", os.path.join(rocm, "include"),
                        os.path.join(HERE, "span_rules.cpp"), "-o", str(exe)],
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    r = subprocess.run([str(exe)], capture_output=True, text=True, timeout=60)
    assert r.returncode == 0 and "all checks passed" in r.stdout, r.stdout + r.stderr


@pytest.mark.parametrize("shift,refused", [(0, False),  # in place
                                           (4, True), (31, True), (32, False),
                                           (64, False), (96, False), (97, True), (127, True)])
def test_slices_of_one_buffer_in_a_plan(shift, refused):
    """32 columns of rows 128 elements apart, beside the input's: what shares memory is
    refused, and what does not goes past the check (a plan touches no operand)."""
    if build.is_stale():
        build.build()
    at = 1 << 40
    status = _lib.LAMB_OK
    try:
        _ops.lamb_ortho_plan_create([(at, at + 4 * shift, 10, 32, 128, 128)], 0, 0, 1).close()
    except _lib.LambError as e:
        status = e.status
    assert (status == _lib.LAMB_EOVERLAP) == refused
