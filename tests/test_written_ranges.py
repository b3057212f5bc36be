"""The check of a call's buffers for overlaps (CPU).

csrc/written_ranges.h is host code without HIP; tests/written_ranges_check.cpp
drives it beside a comparison of every pair.
"""
import os
import shutil
import subprocess

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(os.path.dirname(HERE), "paper_2412_07210_amd", "csrc")


def test_finds_what_comparing_every_pair_finds(tmp_path):
    cxx = shutil.which("g++") or shutil.which("c++")
    if cxx is None:
        pytest.skip("no C++ compiler")
    program = str(tmp_path / "check")
    subprocess.run([cxx, "-O1", "-std=c++17", "-Wall", "-fsanitize=undefined", "-fno-sanitize-recover=all", "-I", CSRC,
                    os.path.join(HERE, "written_ranges_check.cpp"), "-o", program], check=True)
    r = subprocess.run([program], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0, r.stdout + r.stderr
    counts = [int(x) for x in r.stdout.split()]
    assert len(counts) == 5 and min(counts) > 10_000
