"""Which blocks a windowed walk reads, on the host: csrc/window.hpp, which the kernels, their
plan and their tile map use, built by g++ and driven over all small calls. A caller may give up
the memory of blocks behind a window, so a stale id there must never be followed; on the
GPU that cannot be seen from values, since what is read there is masked."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2608_23658_amd", "csrc")


def test_walks_begin_at_the_block_of_the_first_key_seen(tmp_path):
    gxx = shutil.which("g++")
    if gxx is None:
        pytest.skip("g++ not available")
    exe = str(tmp_path / "window_walks")
    r = subprocess.run([gxx, "-std=c++17", "-O1", "-Wall", "-Werror", "-I", CSRC,
                        os.path.join(ROOT, "tests", "window_walks.cpp"), "-o", exe],
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    r = subprocess.run([exe], capture_output=True, text=True, timeout=60)
    assert r.returncode == 0 and r.stdout.startswith("ok:"), r.stdout + r.stderr
