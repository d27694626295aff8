"""The host checks of the operators beside the round again, against the library's host code built with
AddressSanitizer and UndefinedBehaviorSanitizer (any finding aborts)."""
import os
import subprocess
import sys

import pytest

from test_abi_sanitized import HERE, ROOT, _clang_asan_runtime


def test_train_host_tests_pass_under_sanitizers(tmp_path):
    rt = _clang_asan_runtime()
    if rt is None:
        pytest.skip("clang's AddressSanitizer runtime is not installed")
    from paper_2205_14473_amd.build import build_host_sanitized
    try:
        lib = build_host_sanitized(str(tmp_path / "san"))
    except FileNotFoundError as e:
        pytest.skip(str(e))
    env = dict(os.environ, EA_LIB=lib)
    env["LD_PRELOAD"] = " ".join([rt] + ([env["LD_PRELOAD"]] if env.get("LD_PRELOAD") else []))
    env["ASAN_OPTIONS"] = "detect_leaks=0:abort_on_error=1:verify_asan_link_order=0"
    env["UBSAN_OPTIONS"] = "print_stacktrace=1:halt_on_error=1"
    r = subprocess.run([sys.executable, "-m", "pytest", "-q", "-x", "-p", "no:cacheprovider", "-m", "not gpu",
                        "-k", "not host_tensors", os.path.join(HERE, "test_train_host.py")],
                       cwd=ROOT, env=env, capture_output=True, text=True, timeout=900)
    out = r.stdout + r.stderr
    assert r.returncode == 0, out[-4000:]
    assert "runtime error" not in out and "AddressSanitizer" not in out, out[-4000:]
    assert " passed" in out
