"""The serving entry points' host code under AddressSanitizer (no GPU needed), as
tests/test_abi_asan_cpu.py does it for the others: their argument checks run in a child
Python against a library whose host code is instrumented."""

import os
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_serving_error_paths_under_asan(tmp_path):
    sys.path.insert(0, ROOT)
    from tests import asan_build

    try:
        rt = asan_build.asan_runtime()
    except FileNotFoundError as e:  # pragma: no cover
        pytest.skip(str(e))
    lib = asan_build.build_asan(str(tmp_path / "asan"))
    env = dict(os.environ)
    env.update(LD_PRELOAD=rt, DUO_TEST_LIB=lib, ASAN_OPTIONS="detect_leaks=0:abort_on_error=1:halt_on_error=1",
               PYTHONDONTWRITEBYTECODE="1")
    r = subprocess.run([sys.executable, "-m", "pytest", "-q", "-x", "-p", "no:cacheprovider",
                        *(os.path.join(ROOT, "tests", f) for f in ("test_serve_abi_cpu.py", "test_serve_limits_cpu.py"))],
                       cwd=ROOT, env=env, capture_output=True, text=True, timeout=600)
    out = r.stdout + r.stderr
    assert "AddressSanitizer" not in out, out[-4000:]
    assert r.returncode == 0, out[-4000:]
    assert " passed" in r.stdout and "skipped" not in r.stdout
