"""The experts' tile search on the host, lane by lane: every tile of every plan
once, and none for a number past the last."""
import os
import shutil
import subprocess

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(os.path.dirname(HERE), "paper_1710_02368_amd", "csrc")


def test_tiles_are_found_once(tmp_path):
    if shutil.which("g++") is None:
        pytest.skip("no C++ compiler")
    exe = str(tmp_path / "row_tiles_checks")
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Wno-unknown-pragmas", "-Wno-maybe-uninitialized", "-I", CSRC,
                    os.path.join(HERE, "host_wave", "row_tiles_checks.cpp"), "-o", exe], check=True)
    r = subprocess.run([exe], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0 and ", 0 failure(s)" in r.stdout, r.stdout + r.stderr
