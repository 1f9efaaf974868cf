"""Calls of the recurrence, the residual block and dropout whose launch fails: the runtime's error with its text, and nothing of it left
for the next call.  On the host: a child process that sees no device, whose every launch fails before it reads an address."""
import os
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CODE = """
import ctypes
from paper_2607_19378_b200 import hyenand as hn
L = hn.lib()
runtime = ctypes.CDLL([l.split()[-1] for l in open("/proc/self/maps") if "libcudart" in l][0])
none = runtime.cudaFree(None)                    # what this process gets without a device
assert none != 0
runtime.cudaGetErrorString.restype = ctypes.c_char_p
text = runtime.cudaGetErrorString(none).decode()
runtime.cudaGetLastError()
nothing = runtime.cudaPeekAtLastError()          # 0; without a driver that error stays whatever one does
A = [(i + 1) << 32 for i in range(20)]
def block(C, T, backward):
    head = [2, C, T, 0] + A[:2] + [None] + A[2:5] + [1e-6, 0, 0.0, None, 0]
    if backward: return L.hyenand_block_backward(*head, *A[5:8], A[8], A[9], None, *A[10:13], A[13], None)
    return L.hyenand_block_forward(*head, A[5], A[6], A[7], None)
def recurrence(B, C, n, backward):
    if backward: return L.hyenand_recurrence_backward(B, C, n, 1, 1, *A[:4], None, *A[4:6], None, *A[6:10], None, A[10], None)
    return L.hyenand_recurrence_forward(B, C, n, 1, 1, *A[:4], None, None, A[4], None, None, A[5], None)
calls = {f"block {C} {T} {b}": (lambda C=C, T=T, b=b: block(C, T, b)) for C in (8, 40, 300, 900, 5000) for T in (40, 41) for b in (False, True)}
calls.update({f"recurrence {s} {b}": (lambda s=s, b=b: recurrence(*s, b)) for s in ((2, 3, 20), (2, 300, 9000), (1, 3, 40000), (3, 700, 2500)) for b in (False, True)})
calls["step"] = lambda: L.hyenand_recurrence_step(2, 3, 1, 0, *A[:4], A[4], None, A[5], A[4], None)
calls["dropout"] = lambda: L.hyenand_dropout(1000, 0, A[0], 0.5, A[1], 0, A[2], None)
for name, call in calls.items():
    code, left = call(), runtime.cudaPeekAtLastError()
    assert (code, left) == (hn.HYENAND_ERR_CUDA, nothing) and text in hn.hyenand_last_error(), (name, code, left, hn.hyenand_last_error())
print("fine", len(calls))
"""


def test_a_failed_launch_is_the_calls_own():
    from paper_2607_19378_b200.build import build
    build()
    if os.environ.get("HYENAND_LIB") == "debug":
        pytest.skip("that build talks to the device in front of every launch")
    r = subprocess.run([sys.executable, "-c", CODE], cwd=ROOT, env=dict(os.environ, CUDA_VISIBLE_DEVICES=""), capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and "fine 30" in r.stdout, (r.stdout, r.stderr[-3000:])
