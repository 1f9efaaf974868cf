"""What the residual block has dropped is zero, whatever the gate was there: infinities and NaN in dropped places reach no result, of the
forward or of the gradient.  Every result has the bits of a run with ordinary values in those places."""
import pytest
import torch

from oracle import block as ob
from test_gpu_block import DTYPES, RNG, inputs, run

pytestmark = pytest.mark.gpu


# one CTA, a cluster, more channels than one holds; rows on 16-byte boundaries and not
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("gate", ["none", "sigmoid", "silu"])
@pytest.mark.parametrize("post,pre", [(True, True), (False, True), (True, False), (False, False)])
@pytest.mark.parametrize("B,C,T", [(2, 20, 40), (1, 300, 33), (2, 90, 24), (1, 2100, 33), (1, 2200, 40)], ids=str)
def test_nothing_comes_of_dropped_places(B, C, T, post, pre, gate, dtype):
    t = inputs(B, C, T, DTYPES[dtype], gate, post, True, pre, 1 + C + T)
    gone = ~torch.from_numpy(ob.keep(B * C * T, 0.4, *RNG, 2)).view(B, C, T)
    want = run(t, B, C, T, DTYPES[dtype], gate, 0.4, 2)
    for name, v in want.items():
        assert bool(torch.isfinite(v).all()), name
    which = (["z"] if gate != "none" else []) + ([] if post else ["m"])      # (the norm of m is formed before anything is dropped)
    for value in (float("inf"), float("nan"), -float("inf"), torch.finfo(DTYPES[dtype]).max):
        for n in which:
            bad = dict(t, **{n: t[n].masked_fill(gone, value)})
            got = run(bad, B, C, T, DTYPES[dtype], gate, 0.4, 2)
            for name, v in got.items():
                assert torch.equal(v, want[name]), (n, value, name)
