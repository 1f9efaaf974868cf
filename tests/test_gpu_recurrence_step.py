"""Single tokens of the recurrence against 64 bits, one and thousands of them.

Bound of a step, in units of 2^-24 (u = k v in fp32): 1 of the new state for its one rounding; k v 1; and what else is rounded is of the
smaller side of the decay only, min(a, 1 - a) |s| + |u|, to which the exponential contributes 4 (two steps of the last place), 1 + e and
the quotient 1 each, the inner product and sum 1: 7 in all, and 1 more for the product k v.  An error of the state before is multiplied by a.
y adds the product's rounding and half a step of its type."""
import numpy as np
import pytest
import torch

import oracle
from oracle import recurrence as orec
from test_gpu_recurrence import DTYPES, HALF

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
GATES = {"log": [-1e-6, -3e-5, -1e-3, -0.02, -0.5, -0.69, -0.7, -2.0, -30.0, 0.0], "sigmoid": [12.0, 16.5, 5.0, 1.0, 0.0, -0.5, -3.0, -20.0, 40.0],
         "value": [1.0, 0.999, 0.5, 0.1, -0.9, 0.0, 1.001]}


def walk(decay, dtype, steps, driven):
    from paper_2607_19378_b200 import hyenand as hn
    gates, B, C = GATES[decay], 2, 40 * len(GATES[decay])
    gen = torch.Generator().manual_seed(steps)
    q, k, v = (torch.randn((B, C), generator=gen).to(dtype) for _ in range(3))
    if not driven:
        k.zero_()
    g = torch.tensor(gates).repeat_interleave(40).expand(B, C).contiguous().to(dtype)
    s = torch.randn((B, C), generator=gen)
    state, op = s.cuda(), hn.Recurrence(1, B, C, decay, dtype)
    dev = [t.cuda() for t in (q, k, v, g)]
    for _ in range(steps):
        y = op.step(*dev, state)
    g64 = oracle.to_f64(g)
    a, _ = orec.decay(g64, decay)
    na = {"log": lambda t: -np.expm1(t), "sigmoid": lambda t: 1.0 / (1.0 + np.exp(t)), "value": lambda t: 1.0 - t}[decay](g64)       # 1 - a
    small = np.zeros_like(a) if decay == "value" else np.minimum(a, np.abs(na))
    u, ref, err = oracle.to_f64(k) * oracle.to_f64(v), oracle.to_f64(s), np.zeros((B, C))
    for _ in range(steps):
        before = np.abs(ref) + err
        ref = np.where(np.abs(a) < 0.5, a * ref, ref - na * ref) + u             # (either cancels where the other does not)
        err = np.abs(a) * err + U * (np.abs(ref) + 7 * (small * before + np.abs(u)) + np.abs(u)) * (1 + 1e-6) + 1e-37
    assert np.max(np.abs(oracle.to_f64(state.cpu()) - ref) / err) <= 1.0
    half, want = HALF[dtype], oracle.to_f64(q) * ref
    bound = half * np.abs(want) + (1 + half) * (np.abs(oracle.to_f64(q)) * err + U * np.abs(want)) + 1e-37
    assert np.max(np.abs(oracle.to_f64(y.cpu()) - want) / bound) <= 1.0


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("decay", ["value", "log", "sigmoid"])
@pytest.mark.parametrize("driven", [True, False])
@pytest.mark.parametrize("steps", [1, 2000])
def test_steps(steps, driven, decay, dtype):
    walk(decay, DTYPES[dtype], steps, driven)


@pytest.mark.parametrize("decay,gate", [("value", 0.9), ("log", -0.1), ("log", -3.0), ("sigmoid", 2.0), ("sigmoid", -2.0), ("log", -float("inf")), ("sigmoid", float("inf"))])
def test_states_that_are_not_finite(decay, gate):
    """An infinite state stays one under a decay above 0, a NaN a NaN; a gate of minus infinity forgets, one of plus infinity keeps."""
    from paper_2607_19378_b200 import hyenand as hn
    B, C = 1, 4
    one = torch.ones((B, C), device="cuda")
    state = torch.tensor([[float("inf"), -float("inf"), float("nan"), 2.0]], device="cuda")
    hn.Recurrence(1, B, C, decay).step(one, one, one, one * gate, state)
    a = {"value": lambda t: t, "log": np.exp, "sigmoid": lambda t: 1 / (1 + np.exp(-t))}[decay](np.float64(gate))
    got = state.cpu().double()[0]
    assert bool(got[2].isnan()) and abs(float(got[3]) - (2 * a + 1)) < 1e-6
    if a > 0:
        assert float(got[0]) == float("inf") and float(got[1]) == -float("inf")
    else:
        assert bool(got[:2].isnan().all())                   # (zero times infinity, as the formula has it)
