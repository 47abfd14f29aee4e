"""The argument checks of the operators around the layer (norm, scored routing, gradient norm, 8-bit
products) under AddressSanitizer and UndefinedBehaviorSanitizer: every case of tests/test_block_abi.py
against the sanitized build (CPU only)."""
import os
import subprocess
import sys

from tests.test_host_sanitizers import ROOT, san_env  # noqa: F401


def test_block_abi_cases_clean_under_sanitizers(san_env):  # noqa: F811
    tmp, env = san_env
    cmd = [sys.executable, "-m", "pytest", os.path.join(ROOT, "tests", "test_block_abi.py"), "-q", "-x",
           "-p", "pmpe_san_swap", "-p", "no:cacheprovider", "-m", "not gpu"]
    r = subprocess.run(cmd, env=env, cwd=ROOT, capture_output=True, text=True, timeout=600)
    out = r.stdout + r.stderr
    assert r.returncode == 0, out[-4000:]
    assert "ERROR: AddressSanitizer" not in out and "runtime error:" not in out, out[-4000:]
    assert int(out.split(" passed")[0].split()[-1]) >= 100, out[-2000:]
