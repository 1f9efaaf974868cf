"""A NaN in the residual block's gate shows in every result that it takes part in, and in no other."""
import pytest
import torch

from test_gpu_block import DTYPES, inputs, run

pytestmark = pytest.mark.gpu


# one CTA, a cluster, more channels than one holds
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("gate", ["sigmoid", "silu"])
@pytest.mark.parametrize("post,pre", [(False, False), (True, False), (False, True), (True, True)])
@pytest.mark.parametrize("B,C,T", [(2, 20, 40), (1, 300, 33), (1, 2100, 33)], ids=str)
def test_nan_in_the_gate(B, C, T, post, pre, gate, dtype):
    t = inputs(B, C, T, DTYPES[dtype], gate, post, True, pre, C + T)
    want = run(t, B, C, T, DTYPES[dtype], gate, 0.0)
    at = (B - 1, 7, 13)
    t["z"][at] = float("nan")
    got = run(t, B, C, T, DTYPES[dtype], gate, 0.0)
    element, token = torch.zeros(B, C, T, dtype=torch.bool), torch.zeros(B, C, T, dtype=torch.bool)
    element[at] = True
    token[B - 1, :, 13] = True
    channel, channels = torch.arange(C) == 7, torch.ones(C, dtype=torch.bool)
    # n is the whole token's; behind a norm the gradients are, too
    nan = {"r": element, "n": token, "dx": token if pre else ~channels[None, :, None].expand(B, C, T), "dm": token if pre or post else element,
           "dz": token if pre else element, "dscale": channels if pre else channel, "dg_post": channels if pre else channel, "dg_pre": channels}
    for name, v in got.items():
        assert bool(v[nan[name]].isnan().all()), name
        assert torch.equal(v[~nan[name]], want[name][~nan[name]]), name
