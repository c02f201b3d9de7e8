"""The 4-bit cache's host code (argument checks, launch planning, workspace sizes) under
AddressSanitizer and UndefinedBehaviorSanitizer: the refusal tests of test_cache4_cpu.py in a
child process that loads the sanitized library (CPU only)."""
import os
import subprocess
import sys

import pytest

from tests.test_host_sanitizers import ROOT, _gpu_visible


@pytest.mark.skipif(_gpu_visible(), reason="a host-only check; runs where no GPU is visible")
def test_refusals_are_clean_under_asan_and_ubsan():
    from paper_2609_22158_amd.build import build_host_sanitized, sanitizer_env

    build_host_sanitized()
    env = sanitizer_env()
    env["PYTHONPATH"] = ROOT + os.pathsep + env.get("PYTHONPATH", "")
    r = subprocess.run([sys.executable, "-m", "pytest", "-q", "-p", "no:cacheprovider",
                        os.path.join(ROOT, "tests", "test_cache4_cpu.py"),
                        "-k", "refuse or workspace or nothing or exports or needs"],
                       cwd=ROOT, env=env, capture_output=True, text=True, timeout=900)
    out = r.stdout + r.stderr
    assert r.returncode == 0, out[-6000:]
    assert "passed" in out and "runtime error" not in out and "AddressSanitizer" not in out
