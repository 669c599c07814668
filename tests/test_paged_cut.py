"""How attention over pages is cut: the integer work the kernels do, run on the CPU.  Every token a query sees is in one tile, every tile in one
share, every part of a cut sequence has a slot of its own, and every query tile of a ragged batch has a place."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.skipif(shutil.which("g++") is None, reason="no host compiler")
def test_tiles_shares_and_places(tmp_path):
    exe = str(tmp_path / "paged_cut_drive")
    build = subprocess.run(["g++", "-std=c++17", "-O2", "-Wall", "-Wno-unknown-pragmas", "-o", exe, os.path.join(ROOT, "tests", "paged_cut_drive.cpp")],
                           capture_output=True, text=True)
    assert build.returncode == 0, build.stderr[-4000:]
    run = subprocess.run([exe], capture_output=True, text=True, timeout=300)
    assert run.returncode == 0 and "ok" in run.stdout, (run.stdout[-2000:], run.stderr[-2000:])
