"""The recurrence, the residual block and dropout against the checked build: every access to global memory compared with the ranges of
its call (tests/conftest.py fails any test after which one was outside)."""
import os
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
# (tensors of more than 2^31 elements take minutes there and add no kernel; that build synchronises in every call, which a capture
# does not allow)
SKIP = "not beyond_32_bits and not captured and not at_once"


@pytest.mark.gpu
def test_no_access_outside_the_ranges_of_a_call():
    if os.environ.get("HYENAND_LIB") == "debug":
        pytest.skip("running against the checked build")
    r = subprocess.run([sys.executable, "-m", "pytest", "-m", "gpu", "-x", "-q", "-p", "no:cacheprovider", "-k", SKIP,
                        "tests/test_gpu_recurrence.py", "tests/test_gpu_block.py", "tests/test_gpu_layer.py"],
                       cwd=ROOT, env=dict(os.environ, HYENAND_LIB="debug"), capture_output=True, text=True, timeout=1500)
    assert r.returncode == 0, (r.stdout[-3000:], r.stderr[-2000:])
