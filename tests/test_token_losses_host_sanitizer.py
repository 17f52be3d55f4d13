"""The CPU tests of the token losses and 4-bit rows' entry points against the build whose host code carries
AddressSanitizer and UndefinedBehaviorSanitizer (device code untouched): no refusal, size or message may
trip either."""
import os
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.timeout(600)
def test_entry_points_under_host_sanitizers():
    from paper_1804_06087_amd import build_sanitized as bs
    env = bs.env_for(bs.build_sanitized())
    r = subprocess.run([sys.executable, "-m", "pytest", "-x", "-q", "-p", "no:cacheprovider", "-m", "not gpu",
                        "tests/test_token_losses_cpu.py"], cwd=ROOT, env=env, capture_output=True, text=True, timeout=540)
    out = r.stdout + r.stderr
    assert r.returncode == 0, out[-4000:]
    assert "AddressSanitizer" not in out and "runtime error:" not in out, out[-4000:]
    assert " passed" in out
