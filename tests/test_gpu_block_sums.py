"""The residual block's sums where one token or one channel is all there is: a remainder that a tile, a warp or a slot of the workspace
left out would change the result by all of it.

Bound: the element's own roundings as in test_gpu_block.py without its term for many addends (a sum of one number and zeros is exact),
K = 100 of 2^-24."""
import numpy as np
import pytest
import torch

import oracle
from oracle import block as ob
from test_gpu_block import DTYPES, EPS, HALF, inputs, run

pytestmark = pytest.mark.gpu

K = 100


def compare(got, ref, names):
    for k in names:
        half = HALF[got[k].dtype]
        bound = half * np.abs(ref[k]) + K * 2.0 ** -24 * ref[k + "_abs"] * (1 + half) + 1e-37
        worst = np.max(np.abs(oracle.to_f64(got[k]) - ref[k]) / bound)
        assert np.isfinite(worst) and worst <= 1.0, f"{k}: an element is off by {worst:.2f} x its bound"


# more tiles than the backward has slots, a last tile of one token; one CTA, clusters, more channels than a cluster holds
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("B,C,T", [(3, 5, 20001), (2, 8, 40000), (1, 24, 20033), (2, 40, 20001), (1, 300, 20001), (2, 90, 40004), (1, 768, 4097), (1, 1500, 2049), (40, 130, 33),
                                   (2, 2100, 65), (1, 5000, 129)], ids=str)
def test_one_token_of_all(B, C, T, dtype):
    """Gradients at one token: the last, the first, one between; the sums over tokens are that token's."""
    t = inputs(B, C, T, DTYPES[dtype], "silu", True, True, True, B + T)
    for b, at in ((B - 1, T - 1), (0, 0), (B // 2, T // 2 + 1), (B - 1, max(0, T - 32)), (0, T - 2)):
        one = {k: torch.zeros_like(t[k]) for k in ("dr", "dn")}
        for k in one:
            one[k][b, :, at] = t[k][b, :, at]
        got = run(dict(t, **one), B, C, T, DTYPES[dtype], "silu", 0.0)
        cut = lambda x: x[b:b + 1, :, at:at + 1]
        ref = ob.block(cut(t["x"]), cut(t["m"]), cut(t["z"]), t["g_post"], t["scale"], t["g_pre"], EPS, "silu", None, cut(t["dr"]), cut(t["dn"]))
        # (means over C channels stand in every term)
        for k in ("dg_post", "dscale", "dg_pre"):
            bound = (K + C) * 2.0 ** -24 * ref[k + "_abs"] + 2.0 ** -24 * np.abs(ref[k]) + 1e-37
            assert np.all(np.abs(oracle.to_f64(got[k]) - ref[k]) <= bound), k


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("C,T", [(5, 33), (24, 40), (40, 33), (90, 64), (300, 31), (768, 72), (1030, 21), (1500, 33), (2048, 40), (2100, 33), (5000, 36)], ids=str)
def test_one_channel_of_all(C, T, dtype):
    """All of a token in one channel, another for every token: both norms and both means are that channel's."""
    B = 1
    t = inputs(B, C, T, DTYPES[dtype], "silu", True, True, True, C)
    at = (torch.arange(T) * 7 + C - 1) % C
    at[0], at[1] = C - 1, 0
    only = torch.zeros((B, C, T), dtype=torch.bool)
    only[0, at, torch.arange(T)] = True
    for k in ("x", "m", "dr", "dn"):
        t[k] = torch.where(only, t[k], torch.zeros_like(t[k]))
    got = run(t, B, C, T, DTYPES[dtype], "silu", 0.0)
    ref = ob.block(t["x"], t["m"], t["z"], t["g_post"], t["scale"], t["g_pre"], EPS, "silu", None, t["dr"], t["dn"])
    compare(got, ref, ("r", "n", "dx", "dm", "dz"))
