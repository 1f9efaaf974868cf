"""Tiles of the residual block's forward that meet twice: the branch cancels most of x, or its squares before the norm are beyond fp32.

Bound of an element: that of test_gpu_block.py, K 2^-24 of the absolute terms with K = 100 + C, and half a step of the result's type.
A tile that met once only would miss it: with x = -(1 - 2^-12) branch the sum of r^2 is 2^-24 of the squares that it would be the
difference of, all of which rounding takes; with squares beyond fp32 n would be 0."""
import numpy as np
import pytest
import torch

import oracle
from oracle import block as ob
from test_gpu_block import DTYPES, EPS, HALF, RNG, inputs, run

pytestmark = pytest.mark.gpu


def check(t, B, C, T, dtype, gate, p=0.0, site=0):
    got = run(t, B, C, T, DTYPES[dtype], gate, p, site)
    D = ob.factor((B, C, T), p, RNG, site) if p else None
    ref = ob.block(t["x"], t["m"], t["z"], t["g_post"], t["scale"], t["g_pre"], EPS, gate, D, t["dr"], t["dn"])
    for k, v in got.items():
        half = HALF[v.dtype]
        K = 100 + C + (64 + B * T / 32 if v.dim() == 1 else 0)
        bound = half * np.abs(ref[k]) + K * 2.0 ** -24 * ref[k + "_abs"] * (1 + half) + 1e-37
        worst = np.max(np.abs(oracle.to_f64(v) - ref[k]) / bound)
        assert np.isfinite(worst) and worst <= 1.0, f"{k}: an element is off by {worst:.2f} x its bound"


# one CTA with wide tiles, one with narrow ones, clusters of two to eight; rows on 16-byte boundaries and not; several tiles a cluster
SHAPES = [(2, 20, 48), (1, 90, 33), (2, 300, 64), (2, 300, 31), (1, 768, 72), (3, 768, 210), (1, 1500, 33), (1, 2048, 40), (300, 300, 9)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("B,C,T", SHAPES, ids=str)
def test_a_branch_that_cancels_the_stream(B, C, T, dtype):
    """In every other tile, so that meetings of one and of two follow each other; with and without the norm of m."""
    for post, p in ((True, 0.0), (False, 0.2)):
        t = inputs(B, C, T, DTYPES[dtype], "silu", post, True, True, 100 + C + T)
        D = ob.factor((B, C, T), p, RNG, 0) if p else None
        zero = torch.zeros_like(t["x"])
        branch = torch.from_numpy(ob.block(zero, t["m"], t["z"], t["g_post"], t["scale"], None, EPS, "silu", D)["r"])
        some = (torch.arange(T) // 32 % 2 == 0)[None, None] & (torch.arange(B) % 3 != 1)[:, None, None]
        t["x"] = torch.where(some & (branch != 0), -(1 - 2.0 ** -12) * branch, t["x"].double()).to(DTYPES[dtype])
        check(t, B, C, T, dtype, "silu", p)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("B,C,T", SHAPES + [(1, 3, 8), (1, 2100, 33)], ids=str)
def test_squares_beyond_fp32(B, C, T, dtype):
    """m at 1e17 and an open gate of 100: b^2 is infinite, r is not."""
    t = inputs(B, C, T, DTYPES[dtype], "silu", True, True, True, C + T)
    t["m"], t["z"] = (t["m"].float() * 1e17 / 3).to(DTYPES[dtype]), torch.full_like(t["z"], 100.0)
    t["m"][:, :, 1::5] *= 1e-17
    check(t, B, C, T, dtype, "silu")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("B,C,T", SHAPES, ids=str)
def test_tokens_do_not_change_their_neighbours(B, C, T, dtype):
    """A token that cancels, or holds a NaN, sends its tile into the second meeting: the others keep their bits."""
    t = inputs(B, C, T, DTYPES[dtype], "silu", True, True, True, 7 + C + T)
    want = run(t, B, C, T, DTYPES[dtype], "silu", 0.0)
    branch = torch.from_numpy(ob.block(torch.zeros_like(t["x"]), t["m"], t["z"], t["g_post"], t["scale"], None, EPS, "silu")["r"])
    other = torch.arange(T) % 3 == 1
    for change in ((-(1 - 2.0 ** -12) * branch).to(DTYPES[dtype]), torch.full_like(t["x"], float("nan")), torch.full_like(t["x"], 3e19)):
        got = run(dict(t, x=torch.where(other, change, t["x"])), B, C, T, DTYPES[dtype], "silu", 0.0)
        for name in ("r", "n", "dx", "dm", "dz"):
            assert torch.equal(got[name][:, :, ~other], want[name][:, :, ~other]), name
