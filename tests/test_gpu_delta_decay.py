"""Decays of the delta rule at both ends: so slow that a state outlives a whole sequence, against the closed form.

Bound: a state is rounded once in every chunk of 64 tokens, by at most 2^-25 of it on average, and with either sign as what is taken off it
differs from chunk to chunk: sqrt(4096) 2^-25 = 1.9e-6 for 262144 tokens.  In segments the map of each has the rounding of its own chunks,
the same in all of them where all decays are equal: 74 sqrt(56) 2^-25 = 1.7e-5 for two heads; held to these.  gamma_64 as a factor is off by
the same half step in every chunk: 4096 2^-25 = 1.2e-4 at worst, 7e-5 to 1.6e-4 at these decays."""
import numpy as np
import pytest
import torch

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
