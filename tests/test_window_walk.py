"""Which tiles attention with a window goes through, on the host: tests/window_walk_check.cpp."""
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_every_visible_pair_is_met_once(tmp_path):
    exe = str(tmp_path / "window_walk_check")
    try:
        r = subprocess.run(["g++", "-std=c++17", "-O2", "-Wall", "-Werror", "-fsanitize=undefined", "-fno-sanitize-recover",
                            os.path.join(ROOT, "tests", "window_walk_check.cpp"), "-o", exe], capture_output=True, text=True)
    except FileNotFoundError:
        pytest.skip("no host compiler")
    assert r.returncode == 0, r.stderr
    r = subprocess.run([exe], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and "0 failure(s)" in r.stdout, r.stdout + r.stderr
