"""The pieces of the queries past the windows in the largest batches, on the host:
tests/window_pieces_check.cpp."""
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_pieces_of_the_largest_batches(tmp_path):
    exe = str(tmp_path / "window_pieces_check")
    try:
        r = subprocess.run(["g++", "-std=c++17", "-O2", "-Wall", "-Werror", "-fsanitize=undefined", "-fno-sanitize-recover",
                            os.path.join(ROOT, "tests", "window_pieces_check.cpp"), "-o", exe], capture_output=True, text=True)
    except FileNotFoundError:
        pytest.skip("no host compiler")
    assert r.returncode == 0, r.stderr
    r = subprocess.run([exe], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and " 0 failure(s)" in r.stdout, r.stdout + r.stderr
