"""The tile lists of the orthogonalised updates' symmetric products (CPU).

csrc/ortho_tiles.h is host code without HIP; tests/ortho_tiles_check.cpp drives
it over 6,000 random layouts.
"""
import os
import re
import shutil
import subprocess

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(ROOT, "paper_2412_07210_amd", "csrc")


def test_every_tile_once_and_pieces_within_the_workspace(tmp_path):
    cxx = shutil.which("g++") or shutil.which("c++")
    if cxx is None:
        pytest.skip("no C++ compiler")
    program = str(tmp_path / "check")
    subprocess.run([cxx, "-O1", "-std=c++17", "-Wall", "-fsanitize=undefined", "-fno-sanitize-recover=all", "-I", CSRC,
                    os.path.join(HERE, "ortho_tiles_check.cpp"), "-o", program], check=True)
    r = subprocess.run([program], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stdout + r.stderr
    whole, cut, limited = (int(x) for x in r.stdout.split())
    assert whole > 500 and cut > 500 and limited > 0


def test_documented_limit_is_the_enforced_one():
    header = open(os.path.join(ROOT, "include", "edit_outer.h")).read()
    code = open(os.path.join(CSRC, "ortho_tiles.h")).read()
    documented = re.search(r"up to (\d+) MiB for unfinished", header)
    assert documented and f"kPieceBytes = int64_t({documented.group(1)}) << 20" in code
