"""Copies of the recurrence that do not come in time: the warp that waited for them stores nothing from there on, what follows from its
positions is NaN, the status word says so, and the next call is whole again.  The checked build takes the copies of one tile to be late
without waiting for anything."""
import os
import subprocess
import sys

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
DEBUG = os.environ.get("HYENAND_LIB") == "debug"
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
LEFT = 7.0                                       # what the outputs held before
checked = pytest.mark.skipif(not DEBUG, reason="the checked build holds the copies back")


def inputs(B, C, L, dtype):
    gen = torch.Generator().manual_seed(L)
    d = {n: torch.randn((B, C, L), generator=gen).to(dtype).cuda() for n in ("q", "k", "v", "g", "dy")}
    d.update({n: torch.randn((B, C), generator=gen).cuda() for n in ("s0", "ds")}, lengths=None)
    return d


def calls(d, B, C, L, dtype, marks=None, tile=-1, warp=-1):
    """y, s_end and dq, dk, dv, dg, ds0, over buffers of LEFT; the gradients from `marks` where they are given."""
    from paper_2607_19378_b200 import hyenand as hn
    code = {torch.float32: 0, torch.bfloat16: 1}[dtype]
    like = lambda t: torch.full_like(t, LEFT)
    o = {"y": like(d["q"]), "s_end": like(d["s0"]), "ds0": like(d["s0"]), **{n: like(d["q"]) for n in ("dq", "dk", "dv", "dg")}}
    mk = torch.zeros((B, C, hn.hyenand_recurrence_marks(L)), device="cuda")
    work = torch.zeros(hn.hyenand_recurrence_workspace_bytes(B, C, L, code), dtype=torch.uint8, device="cuda")
    assert hn.hyenand_debug_recurrence_late(tile, warp) == 0
    try:
        hn.hyenand_recurrence_forward(B, C, L, 2, code, d["q"], d["k"], d["v"], d["g"], d["s0"], d["lengths"], o["y"], o["s_end"], mk, work)
        hn.hyenand_recurrence_backward(B, C, L, 2, code, d["q"], d["k"], d["v"], d["g"], d["lengths"], mk if marks is None else marks, d["dy"], d["ds"],
                                       o["dq"], o["dk"], o["dv"], o["dg"], o["ds0"], work)
        torch.cuda.synchronize()
    finally:
        hn.hyenand_debug_recurrence_late(-1)
    assert tile < 0 or hn.hyenand_recurrence_device_status() == 1
    return o, mk


# lanes of a row forward and backward, 8 positions each, 16 of bf16; rows cut into segments where the last is true
@pytest.mark.gpu
@checked
@pytest.mark.parametrize("B,C,L,dtype,lanes_fwd,lanes_bwd,tile,cut", [
    (2, 5, 1000, "bf16", 64, 64, 0, False), (3, 601, 1536, "bf16", 32, 32, 1, False), (3, 601, 777, "f32", 32, 32, 2, False),
    (3, 601, 2500, "bf16", 64, 64, 1, False), (1, 500, 9000, "bf16", 192, 128, 1, False), (1, 700, 9000, "bf16", 128, 256, 1, False),
    (1, 300, 5000, "f32", 256, 128, 1, False), (1, 3, 40000, "bf16", 32, 32, 20, True), (2, 10, 20011, "f32", 32, 32, 33, True)], ids=str)
def test_all_copies_of_a_tile(B, C, L, dtype, lanes_fwd, lanes_bwd, tile, cut):
    fwd, bwd = (lanes * (8 if dtype == "f32" else 16) for lanes in (lanes_fwd, lanes_bwd))
    d = inputs(B, C, L, DTYPES[dtype])
    want, marks = calls(d, B, C, L, DTYPES[dtype])
    got, _ = calls(d, B, C, L, DTYPES[dtype], marks, tile)
    # a row starts up to seven positions into its first tile
    y, ref = got["y"], want["y"]
    assert torch.equal(y[:, :, :max(0, tile * fwd - 7)], ref[:, :, :max(0, tile * fwd - 7)])
    behind = y[:, :, tile * fwd:]
    assert behind.numel() and bool((behind[:, :, :fwd - 7] == LEFT).all())
    assert bool(((behind == LEFT) | (behind.isnan() if cut else False)).all()) and bool(got["s_end"].isnan().all())
    for n in ("dq", "dk", "dv", "dg"):
        x, ref, at = got[n], want[n], (tile + 1) * bwd
        assert torch.equal(x[:, :, at:], ref[:, :, at:]), n
        x = x[:, :, :max(0, at - 7)]
        assert x.numel() and bool((x[:, :, tile * bwd:] == LEFT).all()), n
        # (dq takes the states alone, which the forward's marks give)
        other = False if not cut else x == ref[:, :, :x.shape[2]] if n == "dq" else x.isnan()
        assert bool(((x == LEFT) | other).all()), n
    assert bool(got["ds0"].isnan().all())
    again, _ = calls(d, B, C, L, DTYPES[dtype])
    assert all(torch.equal(again[n], want[n]) for n in want)


@pytest.mark.gpu
@checked
@pytest.mark.parametrize("B,C,L,dtype,lanes_fwd,lanes_bwd", [(3, 601, 2504, "bf16", 64, 64), (1, 500, 9000, "bf16", 192, 128), (1, 700, 9000, "bf16", 128, 256),
                                                             (1, 300, 5000, "f32", 256, 128)], ids=str)
def test_copies_of_one_warp_of_a_row(B, C, L, dtype, lanes_fwd, lanes_bwd):
    """Warp 1 stores nothing from tile 1 on; the warps that go on from its state, or from its gradient of one, store NaN."""
    per = 8 if dtype == "f32" else 16
    d = inputs(B, C, L, DTYPES[dtype])
    want, marks = calls(d, B, C, L, DTYPES[dtype])
    got, _ = calls(d, B, C, L, DTYPES[dtype], marks, 1, 1)
    at = torch.arange(L, device="cuda")
    tile_f, warp_f = at // (per * lanes_fwd), at // (per * 32) % (lanes_fwd // 32)
    tile_b, warp_b = at // (per * lanes_bwd), at // (per * 32) % (lanes_bwd // 32)
    expected = {"y": ((tile_f >= 1) & (warp_f == 1), (tile_f > 1) | (tile_f == 1) & (warp_f > 1))}
    left = (tile_b <= 1) & (warp_b == 1)
    # (the marks begin every tile anew, but warp 1 fetches nothing for tile 0 either)
    no_state, no_gradient = (tile_b <= 1) & (warp_b > 1), (tile_b < 1) | (tile_b == 1) & (warp_b < 1)
    expected.update(dq=(left, no_state), dk=(left, no_gradient), dv=(left, no_gradient), dg=(left, no_state | no_gradient))
    for n, (left, nan) in expected.items():
        ref = torch.where(left, torch.full_like(want[n], LEFT), torch.where(nan, torch.full_like(want[n], float("nan")), want[n]))
        assert bool(((got[n] == ref) | (got[n].isnan() & ref.isnan())).all()), n
    assert bool(got["s_end"].isnan().all()) and bool(got["ds0"].isnan().all())


@pytest.mark.gpu
def test_with_the_checked_build():
    if DEBUG:
        pytest.skip("running against the checked build")
    r = subprocess.run([sys.executable, "-m", "pytest", "-m", "gpu", "-x", "-q", "-p", "no:cacheprovider", os.path.abspath(__file__)], cwd=ROOT,
                       env=dict(os.environ, HYENAND_LIB="debug"), capture_output=True, text=True, timeout=600)
    assert r.returncode == 0 and "13 passed" in r.stdout, (r.stdout[-3000:], r.stderr[-2000:])


def test_product_library_holds_nothing_back():
    if DEBUG:
        pytest.skip("running against the checked build")
    from paper_2607_19378_b200.build import build
    build()
    from paper_2607_19378_b200 import hyenand as hn
    assert hn.hyenand_debug_recurrence_late(1) == -1 and hn.hyenand_debug_recurrence_late(-1) == -1
