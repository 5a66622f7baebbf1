"""The planner of masked batches under AddressSanitizer and
UndefinedBehaviorSanitizer, on the CPU, as test_host_sanitized.py runs the rest
of the host code."""

import os
import subprocess
import sys

from tests.test_host_sanitized import ROOT, sanitized_env  # noqa: F401

DEVICE_TESTS = "score_options"


def test_masked_plans_under_the_sanitizers(sanitized_env):  # noqa: F811
    r = subprocess.run([sys.executable, "-m", "pytest", "-q", "-p", "no:cacheprovider",
                        os.path.join(ROOT, "tests", "test_host_masks.py"), "-k", f"not {DEVICE_TESTS}"],
                       cwd=ROOT, env=sanitized_env, capture_output=True, text=True, timeout=900)
    assert r.returncode == 0, (r.stdout + r.stderr)[-3000:]
    assert " passed" in r.stdout
