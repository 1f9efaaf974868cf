"""Waits of the delta rule that run out: every kernel returns, what follows from the chunk concerned is NaN and not a plausible number, other
heads and chunks keep their bits, the status word says so, and the next call is whole again.  The checked build takes a wait of head 0 to have
run out without waiting for anything; what it waits for comes all the same."""
import os
import subprocess
import sys

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
DEBUG = os.environ.get("HYENAND_LIB") == "debug"
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
PREPARE, WALK, MAPS, JOIN, BACK, BACK_MAPS, GRADIENTS = range(7)
COPIES, PRODUCT, RESULT = range(3)
checked = pytest.mark.skipif(not DEBUG, reason="the checked build holds the waits")


def calls(t, shape, dtype, forward=(-1, 0, 0), backward=(-1, 0, 0), marks=None):
    """Outputs of both calls, every element NaN or a number of theirs; the gradients from `marks` where they are given."""
    from paper_2607_19378_b200 import hyenand as hn
    B, H, Hk, Dk, Dv, L = shape
    op = hn.DeltaRule(L, B, H, Dk, Dv, Hk, "log", dtype)
    x = [t[n] for n in ("q", "k", "v", "g", "beta")]
    try:
        assert hn.hyenand_debug_delta_late(*forward) == 0
        y, s_end, mk = op.forward(*x, s0=t["s0"], marks=True)
        hn.hyenand_debug_delta_late(*backward)
        grads = op.backward(*x, mk if marks is None else marks, t["dy"], ds_end=t["ds"])
        torch.cuda.synchronize()
    finally:
        hn.hyenand_debug_delta_late(-1)
    assert max(forward[0], backward[0]) < 0 or hn.hyenand_delta_device_status() == 1
    out = dict(zip(("y", "s_end", "dq", "dk", "dv", "dg", "dbeta", "ds0"), (y, s_end) + grads))
    return {n: a.reshape(H, -1, a.shape[-1]) for n, a in out.items()}, mk


def check(got, want, lost, perhaps=None):
    """Head 0: `lost` tokens (or all of a state) are NaN, those of `perhaps` too or as they were, the rest as it was; head 1 as it was."""
    for n, a in got.items():
        w, gone = want[n], lost.get(n, slice(0, 0))
        assert torch.equal(a[1], w[1]), f"{n}: another head"
        nan = torch.zeros(a.shape[-1], dtype=torch.bool, device="cuda")
        nan[gone] = True
        maybe = torch.zeros_like(nan)
        if perhaps is not None and n in perhaps:
            maybe[perhaps[n]] = True
        assert bool(a[0][:, nan].isnan().all()), f"{n}: a number that follows from a lost one"
        same = (a[0] == w[0]) | (a[0].isnan() & maybe)
        assert bool(same[:, ~nan].all()), f"{n}: changed elsewhere"


def problem(shape, dtype):
    sys.path.insert(0, os.path.join(ROOT, "tests"))
    from test_gpu_delta import inputs
    return {n: None if a is None else a.cuda() for n, a in inputs(*shape, dtype, "log", 31).items()}


ALL = slice(None)
TOKENS = ("dk", "dv", "dg", "dbeta")


# tensor copies, threads; one stage and several, with and without room in tensor memory; a chunk in the middle, the first, the last
@pytest.mark.gpu
@checked
@pytest.mark.parametrize("D,L,dtype", [(128, 384, "bf16"), (64, 384, "bf16"), (40, 383, "bf16"), (128, 384, "f32"), (64, 381, "f32")], ids=str)
@pytest.mark.parametrize("c", [2, 0, 5])
def test_one_walk(D, L, dtype, c):
    shape = (1, 2, 2, D, D, L)
    t = problem(shape, DTYPES[dtype])
    want, marks = calls(t, shape, DTYPES[dtype])
    at, to = 64 * c, min(64 * (c + 1), L)
    copied = dtype == "bf16" and L % 8 == 0
    for wait in ([COPIES] if copied else []) + [PRODUCT]:
        got, _ = calls(t, shape, DTYPES[dtype], forward=(PREPARE, c, wait), marks=marks)
        check(got, want, dict(y=slice(at, L), s_end=ALL))
        got, _ = calls(t, shape, DTYPES[dtype], backward=(PREPARE, c, wait))
        check(got, want, dict({n: slice(0, to) for n in TOKENS}, dq=slice(at, to), ds0=ALL))
    for wait in (COPIES, PRODUCT, RESULT):
        got, _ = calls(t, shape, DTYPES[dtype], forward=(WALK, c, wait), marks=marks)
        # (the last result is taken when the state has left)
        check(got, want, dict(y=slice(at, L), s_end=slice(0, 0) if wait == RESULT and to == L else ALL), dict(y=slice(0, at), s_end=ALL))
        got, _ = calls(t, shape, DTYPES[dtype], backward=(BACK, c, wait))
        sure = at if wait == PRODUCT else to                  # (its result may have been taken when the others give up)
        check(got, want, dict({n: slice(0, sure) for n in TOKENS}, ds0=slice(0, 0) if wait == RESULT and c == 0 else ALL),
              dict({n: ALL for n in TOKENS}, ds0=ALL))
    for wait in (COPIES, PRODUCT):
        got, _ = calls(t, shape, DTYPES[dtype], backward=(GRADIENTS, c, wait))
        check(got, want, {n: slice(at, to) for n in ("dq", "dk", "dg", "dbeta")})
    again, _ = calls(t, shape, DTYPES[dtype])
    assert all(torch.equal(again[n], want[n]) for n in want)


# five segments of four chunks: what a segment hands on to the others
@pytest.mark.gpu
@checked
@pytest.mark.parametrize("D,dtype", [(64, "bf16"), (128, "bf16"), (48, "f32")], ids=str)
def test_segments(D, dtype):
    shape = (1, 2, 2, D, D, 1100)
    t = problem(shape, DTYPES[dtype])
    want, marks = calls(t, shape, DTYPES[dtype])
    for kernel, at in ((MAPS, 5), (JOIN, 1)):
        for wait in (COPIES, PRODUCT) if kernel == MAPS else (COPIES,):
            got, _ = calls(t, shape, DTYPES[dtype], forward=(kernel, at, wait), marks=marks)
            check(got, want, dict(y=slice(512, 1100), s_end=ALL))
            got, _ = calls(t, shape, DTYPES[dtype], backward=(BACK_MAPS if kernel == MAPS else JOIN, at, wait))
            check(got, want, dict({n: slice(0, 256) for n in TOKENS}, ds0=ALL))
    got, _ = calls(t, shape, DTYPES[dtype], forward=(WALK, 6, COPIES), marks=marks)        # (a segment's own walk: the others have their states)
    check(got, want, dict(y=slice(384, 512)), dict(y=slice(256, 384)))
    again, _ = calls(t, shape, DTYPES[dtype])
    assert all(torch.equal(again[n], want[n]) for n in want)


@pytest.mark.gpu
def test_with_the_checked_build():
    if DEBUG:
        pytest.skip("running against the checked build")
    r = subprocess.run([sys.executable, "-m", "pytest", "-m", "gpu", "-x", "-q", "-p", "no:cacheprovider", os.path.abspath(__file__)], cwd=ROOT,
                       env=dict(os.environ, HYENAND_LIB="debug"), capture_output=True, text=True, timeout=600)
    assert r.returncode == 0 and "18 passed" in r.stdout, (r.stdout[-3000:], r.stderr[-2000:])


def test_product_library_holds_nothing_back():
    if DEBUG:
        pytest.skip("running against the checked build")
    from paper_2607_19378_b200.build import build
    build()
    from paper_2607_19378_b200 import hyenand as hn
    assert hn.hyenand_debug_delta_late(1, 0, 0) == -1 and hn.hyenand_debug_delta_late(-1) == -1
