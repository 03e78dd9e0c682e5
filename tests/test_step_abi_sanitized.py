"""The host code of the rotation, the windows and the gradient operators under AddressSanitizer and
UndefinedBehaviorSanitizer: compiled for the host only, with
tests/step_abi_host_check.cpp, whose launchers stand in for the kernels'."""
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_step_host_code_under_asan_and_ubsan():
    from paper_2609_36692_amd import _build as B
    if not os.path.exists(B.HIPCC):
        pytest.skip("hipcc not available")
    out = os.path.join(B.OBJ_DIR, "san")
    os.makedirs(out, exist_ok=True)
    exe = os.path.join(out, "step_abi_host_check")
    san = ["-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined",
           "-Xarch_host", "-fno-sanitize-recover=undefined", "-Xarch_host", "-g"]
    srcs = [*(os.path.join(B.CSRC, f) for f in ("np_window_api.cpp", "np_rope_api.cpp", "np_grads_api.cpp")), os.path.join(ROOT, "tests", "step_abi_host_check.cpp")]
    r = subprocess.run([B.HIPCC, "-x", "hip", *B.COMMON, *san, *srcs, "-o", exe], capture_output=True, text=True)
    assert r.returncode == 0, r.stdout + r.stderr
    env = dict(os.environ, ASAN_OPTIONS="halt_on_error=1:detect_leaks=1", UBSAN_OPTIONS="print_stacktrace=1")
    r = subprocess.run([exe], capture_output=True, text=True, env=env, timeout=120)
    log = r.stdout + r.stderr
    assert "AddressSanitizer" not in log and "runtime error" not in log and "LeakSanitizer" not in log, log
    assert r.returncode == 0 and "0 failure(s)" in r.stdout, log
