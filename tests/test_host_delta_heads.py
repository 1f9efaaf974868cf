"""Refusals of the delta rule's and the heads' entry points, without a GPU: addresses are compared and checked on the host before anything is
launched, so plain numbers stand for buffers; and calls whose launch fails."""
import ctypes
import os
import subprocess
import sys

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
A = [(i + 1) << 28 for i in range(24)]           # distinct 16-byte-aligned addresses, 256 MiB apart


@pytest.fixture(scope="module")
def hn():
    from paper_2607_19378_b200.build import build
    build()
    from paper_2607_19378_b200 import hyenand
    return hyenand


def refused(hn, code, word):
    assert code in (hn.HYENAND_ERR_INVALID_ARG, hn.HYENAND_ERR_UNSUPPORTED) and word in hn.hyenand_last_error(), (code, hn.hyenand_last_error())


SHAPES = [(dict(B=0), "must be >= 1"), (dict(H=0), "must be >= 1"), (dict(Hk=0), "must be >= 1"), (dict(Dk=0), "must be >= 1"), (dict(Dv=-1), "must be >= 1"),
          (dict(Hk=3), "no multiple"), (dict(H=2, Hk=4), "no multiple"), (dict(Dk=129), "128 channels"), (dict(Dv=200), "128 channels"),
          (dict(B=1 << 23, H=4, Hk=4), "2^24"), (dict(decay=0), "decay"), (dict(decay=4), "decay"), (dict(dtype=2), "dtype"), (dict(dtype=-1), "dtype"),
          (dict(q=None), "non-NULL"), (dict(k=None), "non-NULL"), (dict(v=None), "non-NULL"), (dict(beta=None), "non-NULL"), (dict(g=None), "exactly where"),
          (dict(decay=3), "exactly where"), (dict(v=A[2] + 8), "aligned"), (dict(g=A[3] + 2), "aligned")]
LONG = [(dict(L=0), "must be >= 1"), (dict(L=(1 << 30) + 1), "2^30"), (dict(B=1 << 10, H=1 << 10, Hk=1, L=1 << 20), "2^36")]
BASE = dict(B=2, H=4, Hk=2, L=40, Dk=16, Dv=24, decay=1, dtype=1, q=A[0], k=A[1], v=A[2], g=A[3], beta=A[4])


@pytest.mark.parametrize("change,word", SHAPES + LONG + [
    (dict(y=None), "y and workspace"), (dict(workspace=None), "y and workspace"), (dict(s0=A[5] + 4), "aligned"), (dict(lengths=A[6] + 2), "aligned"), (dict(y=A[2]), "overlaps"),
    (dict(s_end=A[5] + 16, s0=A[5]), "overlaps"), (dict(marks=A[0]), "overlaps"), (dict(workspace=A[1]), "overlaps"), (dict(workspace=A[9] + 8), "aligned"),
    (dict(lengths=A[7], s_end=A[7]), "overlaps")], ids=str)
def test_delta_forward_refuses(hn, change, word):
    a = dict(BASE, s0=None, lengths=None, y=A[7], s_end=None, marks=None, workspace=A[9], stream=None)
    a.update(change)
    refused(hn, hn.lib().hyenand_delta_forward(*a.values()), word)


@pytest.mark.parametrize("change,word", SHAPES + LONG + [
    (dict(marks=None), "non-NULL"), (dict(dy=None), "non-NULL"), (dict(dq=None), "non-NULL"), (dict(dbeta=None), "non-NULL"), (dict(workspace=None), "non-NULL"),
    (dict(decay=3, g=None), "without a decay"), (dict(dk=A[1]), "overlaps"), (dict(dv=A[7]), "overlaps"), (dict(ds0=A[8] + 16, ds_end=A[8]), "overlaps"),
    (dict(dg=A[13]), "overlaps"), (dict(dy=A[7] + 4), "aligned")], ids=str)
def test_delta_backward_refuses(hn, change, word):
    a = dict(BASE, lengths=None, marks=A[6], dy=A[7], ds_end=None, dq=A[9], dk=A[10], dv=A[11], dg=A[12], dbeta=A[13], ds0=None, workspace=A[14], stream=None)
    a.update(change)
    refused(hn, hn.lib().hyenand_delta_backward(*a.values()), word)


@pytest.mark.parametrize("change,word", SHAPES + [
    (dict(state=None), "non-NULL"), (dict(new_state=None), "non-NULL"), (dict(y=None), "non-NULL"), (dict(y=A[5]), "overlaps"), (dict(new_state=A[5] + 16), "overlaps")],
    ids=str)
def test_delta_step_refuses(hn, change, word):
    a = dict(BASE, state=A[5], active=None, y=A[7], new_state=A[5], stream=None)
    del a["L"]
    a.update(change)
    refused(hn, hn.lib().hyenand_delta_step(*a.values()), word)


HEADS = dict(dims=(6, 8), B=2, Hq=4, Hk=2, D=16, dtype=1, norm=1, axes=(3, 5), base=10000.0, eps=1e-6, q=A[0], k=A[1], g_q=A[2], g_k=A[3], positions=None)


def heads_args(a):
    ints = lambda t: None if t is None else (ctypes.c_int * len(t))(*t)
    a = dict(a)
    dims, axes = a.pop("dims"), a.pop("axes")
    rest = list(a.values())
    return [len(dims), ints(dims)] + rest[:6] + [ints(axes)] + rest[6:]


REFUSED = [(dict(dims=()), "ndim"), (dict(dims=(2, 2, 2, 2), axes=(1, 1, 1, 1)), "ndim"), (dict(dims=(6, 0)), "extent"), (dict(dims=(1 << 20, 1 << 11)), "2^30"),
           (dict(B=0), "must be >= 1"), (dict(Hq=0), "must be >= 1"), (dict(Hk=-1), "must be >= 1"), (dict(D=0), "must be >= 1"), (dict(D=15), "even"), (dict(D=258), "even"),
           (dict(dtype=7), "dtype"), (dict(norm=3), "norm"), (dict(norm=-1), "norm"), (dict(axes=(-1, 2)), "pairs"), (dict(axes=(4, 5)), "pairs"), (dict(base=0.0), "base"),
           (dict(base=float("nan")), "base"), (dict(base=float("inf")), "base"), (dict(eps=0.0), "eps"), (dict(eps=float("nan")), "eps"), (dict(B=1 << 27), "2^28"),
           (dict(q=None), "non-NULL"), (dict(k=None), "non-NULL"), (dict(q=A[0] + 8), "aligned"), (dict(positions=A[5] + 2), "aligned")]


@pytest.mark.parametrize("change,word", REFUSED + [(dict(q_out=None), "non-NULL"), (dict(q_out=A[1]), "overlaps"), (dict(k_out=A[1] + 16), "overlaps"), (dict(k_out=A[7]), "overlaps"),
                                                   (dict(q_out=A[2]), "overlaps")], ids=str)
def test_heads_forward_refuses(hn, change, word):
    a = dict(HEADS, q_out=A[7], k_out=A[8], stream=None)
    a.update(change)
    refused(hn, hn.lib().hyenand_heads_forward(*heads_args(a)), word)


@pytest.mark.parametrize("change,word", REFUSED + [
    (dict(dq_out=None), "non-NULL"), (dict(dk=None), "non-NULL"), (dict(workspace=None), "workspace"), (dict(g_q=None), "not given"), (dict(g_k=None), "not given"),
    (dict(dq=A[0]), "overlaps"), (dict(dq=A[9]), "overlaps"), (dict(dg_q=A[13]), "overlaps"), (dict(workspace=A[10]), "overlaps")], ids=str)
def test_heads_backward_refuses(hn, change, word):
    a = dict(HEADS, dq_out=A[8], dk_out=A[9], dq=A[10], dk=A[11], dg_q=A[12], dg_k=A[13], workspace=A[14], stream=None)
    a.update(change)
    refused(hn, hn.lib().hyenand_heads_backward(*heads_args(a)), word)


def test_sizes(hn):
    assert [hn.hyenand_delta_marks(L, 16, 24) for L in (0, 1, 64, 65, 1 << 30, (1 << 30) + 1)] == [0, 384, 384, 768, (1 << 24) * 384, 0]
    assert hn.hyenand_delta_marks(64, 5, 5) == 8 * 8 and hn.hyenand_delta_marks(64, 129, 1) == 0
    assert hn.hyenand_delta_workspace_bytes(2, 4, 3, 40, 16, 24, 1, 0) == 0 and "multiple" in hn.hyenand_last_error()
    forward, backward = (hn.hyenand_delta_workspace_bytes(2, 4, 2, 40, 16, 24, 1, b) for b in (0, 1))
    assert 8 * 32768 <= forward < backward
    assert hn.hyenand_heads_workspace_bytes(2, (6, 8), 2, 4, 2, 16, 1) >= 2 * 16 * 4 and hn.hyenand_heads_workspace_bytes(2, (6, 8), 2, 4, 2, 15, 1) == 0
    for call in (lambda: hn.hyenand_delta_marks(1 << 32, 16, 16), lambda: hn.hyenand_heads_workspace_bytes(1, ((1 << 32) + 5,), 1, 1, 1, 16, 0)):
        with pytest.raises(OverflowError):
            call()


def test_classes_refuse(hn):
    rule = hn.DeltaRule(8, 2, 4, 6, 10, 2)
    q, v, g = torch.zeros(2, 12, 8), torch.zeros(2, 40, 8), torch.zeros(2, 4, 8)
    with pytest.raises(ValueError, match="q must be"):
        rule.forward(q, q, v, g, g)                          # on the host
    with pytest.raises(ValueError, match="q must be"):
        rule.step(q, q, v, g, g, q)
    with pytest.raises(TypeError, match="q must be a tensor"):
        rule.backward(None, q, v, g, g, q, v)
    for bad in (dict(L=0), dict(B=0), dict(Hk=3), dict(Dk=129), dict(Dv=0), dict(L=(1 << 30) + 1)):
        with pytest.raises(ValueError):
            hn.DeltaRule(**dict(dict(L=8, B=2, H=4, Dk=6), **bad))
    with pytest.raises(KeyError):
        hn.DeltaRule(8, 2, 4, 6, decay="value")
    with pytest.raises(KeyError):
        hn.DeltaRule(8, 2, 4, 6, dtype=torch.float16)
    with pytest.raises(OverflowError):
        hn.DeltaRule((1 << 32) + 8, 2, 4, 6)
    heads = hn.Heads((2, 4), 2, 2, 2, 6, axes=(1, 2))
    x = torch.zeros(2, 12, 2, 4)
    with pytest.raises(ValueError, match="q must be"):
        heads.forward(x, x)
    with pytest.raises(ValueError, match="q must be"):
        heads.backward(x, x, x, x)
    for bad in (dict(dims=(2, 0)), dict(B=0), dict(D=5), dict(D=300, axes=(0, 0)), dict(axes=(2, 2)), dict(axes=(1,)), dict(axes=(-1, 1)), dict(dims=(1, 1, 1, 1), axes=(0, 0, 0, 0))):
        with pytest.raises(ValueError):
            hn.Heads(**dict(dict(dims=(2, 4), B=2, Hq=2, Hk=2, D=6, axes=(1, 2)), **bad))
    with pytest.raises(KeyError):
        hn.Heads((2, 4), 2, 2, 2, 6, norm="layer")


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
A = [(i + 1) << 36 for i in range(20)]
ints = lambda *t: (ctypes.c_int * len(t))(*t)
def delta(H, n, Dk, Dv, dtype, backward):
    head = [2, H, H, n, Dk, Dv, 1, dtype] + A[:5]
    if backward: return L.hyenand_delta_backward(*head, None, A[5], A[6], None, *A[7:12], None, A[12], None)
    return L.hyenand_delta_forward(*head, None, None, A[5], None, None, A[6], None)
def heads(dims, D, dtype, backward):
    head = [len(dims), ints(*dims), 2, 3, 2, D, dtype, 1, None, 1.0, 1e-6] + A[:4] + [None]
    if backward: return L.hyenand_heads_backward(*head, *A[4:10], A[10], None)
    return L.hyenand_heads_forward(*head, A[4], A[5], None)
calls = {f"delta {s} {d} {b}": (lambda s=s, d=d, b=b: delta(*s, d, b)) for s in ((3, 40, 16, 24), (1, 4001, 100, 128), (200, 64, 64, 64)) for d in (0, 1) for b in (False, True)}
calls.update({f"heads {s} {D} {d} {b}": (lambda s=s, D=D, d=d, b=b: heads(s, D, d, b)) for s in ((1,), (33, 5), (64,)) for D in (8, 64, 200) for d in (0, 1) for b in (False, True)})
calls["step"] = lambda: L.hyenand_delta_step(2, 4, 2, 50, 60, 1, 0, *A[:5], A[5], None, A[6], A[5], None)
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
    assert r.returncode == 0 and "fine 49" in r.stdout, (r.stdout, r.stderr[-3000:])
