"""The delta rule's and the heads' tests against the checked build: every access to global memory compared with the ranges of its call
(tests/conftest.py fails any test after which one was outside)."""
import os
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.gpu
def test_no_access_outside_the_ranges_of_a_call():
    if os.environ.get("HYENAND_LIB") == "debug":
        pytest.skip("running against the checked build")
    files = ["delta", "delta_decay", "delta_empty", "delta_layer", "heads", "heads_large"]
    r = subprocess.run([sys.executable, "-m", "pytest", "-m", "gpu", "-x", "-q", "-p", "no:cacheprovider"] + [f"tests/test_gpu_{f}.py" for f in files],
                       cwd=ROOT, env=dict(os.environ, HYENAND_LIB="debug"), capture_output=True, text=True, timeout=1500)
    assert r.returncode == 0, (r.stdout[-3000:], r.stderr[-2000:])
