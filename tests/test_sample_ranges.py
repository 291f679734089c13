"""The ranges of logits that drawn tokens are gathered by (csrc/sample_ranges.h) in a host build: no GPU needed."""

import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def check(tmp_path_factory):
    gxx = shutil.which("g++")
    if not gxx:
        pytest.skip("g++ not available")
    exe = tmp_path_factory.mktemp("ranges") / "sample_ranges_check"
    r = subprocess.run([gxx, "-O1", "-std=c++17", "-Wall", "-Werror",
                        "-I" + os.path.join(ROOT, "paper_2606_12487_amd", "csrc"),
                        os.path.join(ROOT, "tests", "sample_ranges_check.cpp"), "-o", str(exe)],
                       capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr[-2000:]
    return str(exe)


def test_ranges_hold_their_values_and_no_others(check):
    """Every bin, and stretches of bins down to single keys: what a comparison with a range's ends takes is what its
    keys are, none where no fp16 value lies between them; zeros of both signs belong to the bin above them.  Places
    for sorting are in order, and in bounds for any key."""
    r = subprocess.run([check], capture_output=True, text=True, timeout=100)
    assert r.returncode == 0 and r.stdout == "", r.stdout
