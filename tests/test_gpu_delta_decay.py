"""Decays of the delta rule at both ends: so slow that a state outlives a whole sequence, against the closed form; so strong that a head keeps
next to nothing from token to token, against the oracle at the bounds of test_gpu_delta.py.

The gradient of such a decay is as small as the decay itself, while what it could be taken for a difference of (a query's part in a token's
result, a key's part in what is erased and written) stays of order 1: it has to be the sum of what crosses the token, each term of which
carries the decay, so that its relative error is that of its terms.

Bound of the slow ones: a state is rounded once in every chunk of 64 tokens, by at most 2^-25 of it on average, and with either sign as what is taken off it
differs from chunk to chunk: sqrt(4096) 2^-25 = 1.9e-6 for 262144 tokens.  In segments the map of each has the rounding of its own chunks,
the same in all of them where all decays are equal: 74 sqrt(56) 2^-25 = 1.7e-5 for two heads; held to these.  gamma_64 as a factor is off by
the same half step in every chunk: 4096 2^-25 = 1.2e-4 at worst, 7e-5 to 1.6e-4 at these decays."""
import numpy as np
import pytest
import torch

import oracle
from oracle import delta as od
from test_gpu_delta import DTYPES, NAMES, bound as bound_of, compare, inputs, run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("g", [-1e-6, -7e-7, -2e-6])
@pytest.mark.parametrize("H,dtype,bound", [(2, torch.float32, 1.7e-5), (40, torch.float32, 1e-5), (40, torch.bfloat16, 1e-5)], ids=["segments", "f32", "bf16"])
def test_states_that_outlive_a_long_sequence(H, dtype, bound, g):
    from paper_2607_19378_b200 import hyenand as hn
    L, D = 262144, 16
    gen = torch.Generator().manual_seed(1)
    s0, ds = ((1 + torch.rand((1, H, D, D), generator=gen)).cuda() for _ in range(2))
    zero, beta, decay = torch.zeros(1, H * D, L, device="cuda", dtype=dtype), torch.zeros(1, H, L, device="cuda"), torch.full((1, H, L), g, device="cuda")
    op = hn.DeltaRule(L, 1, H, D, dtype=dtype)
    _, s_end, marks = op.forward(zero, zero, zero, decay, beta, s0=s0, marks=True)
    ds0 = op.backward(zero, zero, zero, decay, beta, marks, zero, ds_end=ds)[5]
    left = np.exp(float(np.float32(g)) * L)
    for got, start in ((s_end, s0), (ds0, ds)):
        want = start.double() * left
        assert float((got.double() - want).norm() / want.norm()) <= bound


# one chunk, several, ends inside a chunk; tensor copies and threads; heads that share queries and keys; segments
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape,ragged", [((1, 2, 2, 64, 64, 512), False), ((2, 4, 2, 50, 97, 203), True), ((3, 3, 1, 128, 128, 192), True), ((1, 1, 1, 16, 24, 1096), False),
                                          ((1, 1, 1, 8, 8, 2), False)], ids=str)
@pytest.mark.parametrize("decay,g", [("log", -3.0), ("log", -8.0), ("log", -16.0), ("sigmoid", -16.0), ("log", -30.0)], ids=str)
def test_heads_that_forget(decay, g, shape, ragged, dtype):
    B, H, Hk, Dk, Dv, L = shape
    t = inputs(*shape, DTYPES[dtype], decay, 21, ragged)
    t["g"] = g * (1 + 0.1 * torch.rand((B, H, L), generator=torch.Generator().manual_seed(22)))
    got = run(t, shape, DTYPES[dtype], decay)
    ref = od.delta(t["q"], t["k"], t["v"], t["g"], t["beta"], decay, H, Hk, t["s0"], t["lengths"], t["dy"], t["ds"])
    compare(got, ref, t, H, Hk, DTYPES[dtype], NAMES)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_tokens_that_forget_among_others(dtype):
    """Each of them by itself: beside the others' gradients theirs are 1e-3 to 1e-9."""
    shape = B, H, Hk, Dk, Dv, L = 1, 2, 1, 64, 48, 264
    t = inputs(*shape, DTYPES[dtype], "log", 23)
    at = torch.tensor([0, 1, 15, 16, 17, 40, 63, 64, 65, 100, 127, 130, 200, 255, 256, 263])
    t["g"] *= 0.1
    t["g"][:, :, at] = -6.0 - 14.0 * torch.rand((B, H, len(at)), generator=torch.Generator().manual_seed(24))
    got = run(t, shape, DTYPES[dtype], "log")
    ref = od.delta(t["q"], t["k"], t["v"], t["g"], t["beta"], "log", H, Hk, t["s0"], None, t["dy"], t["ds"])
    compare(got, ref, t, H, Hk, DTYPES[dtype], NAMES)
    # each against |S_{t-1}| |a_t dS|, whose inner product it is
    cut = lambda i, to: [t[n][:, :, i:to] for n in ("q", "k", "v", "g", "beta")] + ["log", H, Hk]
    for i in at.tolist():
        before = oracle.to_f64(t["s0"]) if i == 0 else od.delta(*cut(0, i), t["s0"])["s_end"]
        faded = od.delta(*cut(i, L), before, None, t["dy"][:, :, i:], t["ds"])["ds0"]
        for h in range(H):
            size = np.linalg.norm(before[0, h]) * np.linalg.norm(faded[0, h])
            assert abs(float(got["dg"][0, h, i]) - ref["dg"][0, h, i]) <= bound_of(torch.float32, DTYPES[dtype]) * size, (i, h)
