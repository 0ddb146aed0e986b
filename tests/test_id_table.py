"""The table in LDS that counts a long history's ids (CPU): slices and places of ids are
spread independently, at 3 to 16,000 slices."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.skipif(shutil.which("g++") is None, reason="g++ not available")
def test_slices_and_places(tmp_path):
    exe = str(tmp_path / "id_table")
    subprocess.check_call(["g++", "-std=c++17", "-O2", "-I",
                           os.path.join(ROOT, "paper_2002_06115_amd", "csrc"),
                           os.path.join(ROOT, "tests", "c", "id_table.cpp"), "-o", exe])
    out = subprocess.run([exe], capture_output=True, text=True, timeout=300)
    assert out.returncode == 0, out.stdout + out.stderr
    assert "the table holds" in out.stdout
