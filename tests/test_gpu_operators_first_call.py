"""First calls of a process inside a stream capture (kernels loaded, their limits set and their residency asked there), and first calls of
two threads at once."""
import os
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEAD = """
import threading, torch
from paper_2607_19378_b200 import hyenand as hn
def t(*s): return torch.randn(s, device="cuda")
x, big, w, rng = t(2, 40, 333), t(1, 900, 64), torch.ones(900, device="cuda"), torch.tensor([3, 4], device="cuda")
q, g, one = t(1, 3, 40000), -torch.rand(1, 3, 40000, device="cuda"), torch.ones(40, device="cuda")
def calls():
    rec, long = hn.Recurrence(333, 2, 40, "sigmoid"), hn.Recurrence(40000, 1, 3, "log")
    blk, wide = hn.Block((333,), 2, 40, p=0.2), hn.Block((8, 8), 1, 900)
    out = list(rec.forward(x, x, x, x, marks=True))
    out += list(rec.backward(x, x, x, x, out[2], x))
    l = long.forward(q, q, q, g, marks=True)
    out += list(l) + list(long.backward(q, q, q, g, l[2], q))
    b = blk.forward(x, x, g_post=one, g_pre=one, rng=rng, stats=True)
    out += list(b[:2]) + [o for o in blk.backward(x, x, b[2], g_post=one, g_pre=one, rng=rng, dr=x, dn=x) if o is not None]
    v = big.view(1, 900, 8, 8)
    c = wide.forward(v, v, g_post=w, g_pre=w, stats=True)
    out += list(c[:2]) + [o for o in wide.backward(v, v, c[2], g_post=w, g_pre=w, dr=v, dn=v) if o is not None]
    out += [hn.Dropout(0.3)(x, rng), rec.step(*[x[:, :, 0].contiguous()] * 4, torch.zeros(2, 40, device="cuda"))]
    return out
torch.cuda.synchronize()
"""
CAPTURE = HEAD + """
graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph):
    first = calls()
graph.replay()
torch.cuda.synchronize()
"""
THREADS = HEAD + """
got, streams = [None, None], [torch.cuda.Stream() for _ in range(2)]
def work(i):
    with torch.cuda.stream(streams[i]):
        got[i] = calls()
threads = [threading.Thread(target=work, args=(i,)) for i in range(2)]
for th in threads: th.start()
for th in threads: th.join()
torch.cuda.synchronize()
first = got[0]
assert all(torch.equal(a, b) for a, b in zip(*got))
"""
TAIL = """
# (marks hold one value a piece that a row touches: those behind the last are nobody's)
again = calls()
torch.cuda.synchronize()
assert all(torch.equal(a, b) for i, (a, b) in enumerate(zip(first, again)) if i not in (2, 10))
assert hn.hyenand_recurrence_device_status() == 0 and hn.hyenand_block_device_status() == 0
print("fine")
"""


@pytest.mark.gpu
@pytest.mark.parametrize("code", [CAPTURE, THREADS], ids=["captured", "two threads"])
def test_first_calls(code):
    if os.environ.get("HYENAND_LIB") == "debug":
        pytest.skip("that build synchronises in every call")
    r = subprocess.run([sys.executable, "-c", code + TAIL], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and "fine" in r.stdout, r.stderr[-3000:]
