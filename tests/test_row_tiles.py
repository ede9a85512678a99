"""Which rows each workgroup of the grouped products works on, on the host: the
kernels' own functions with 64 threads as a wave's lanes (tests/row_tiles_check.cpp). A
tile outside the matrix for any offsets, a row missed or done twice for offsets that keep
the rules, or an integer that overflows fails it. No GPU needed."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")
def test_tiles_of_any_offsets(tmp_path):
    exe = str(tmp_path / "row_tiles_check")
    subprocess.run(["g++", "-std=c++17", "-O1", "-g", "-Wno-unknown-pragmas",
                    "-fsanitize=undefined", "-fno-sanitize-recover=all",
                    os.path.join(ROOT, "tests", "row_tiles_check.cpp"), "-o", exe],
                   check=True, capture_output=True, text=True, timeout=300)
    r = subprocess.run([exe], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stdout + r.stderr
    assert "row tiles check ok" in r.stdout
