"""The lines of README.md that use heads and the delta rule, as they stand there, against the oracles."""
import os
import re

import pytest
import torch

import oracle
from oracle import delta as od, heads as oh

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
pytestmark = pytest.mark.gpu


def lines():
    """From the first line of the README that makes heads to the last that uses them or the rule."""
    text = open(os.path.join(ROOT, "README.md")).read().splitlines()
    first = next(i for i, x in enumerate(text) if "hn.Heads(" in x)
    last = max(i for i, x in enumerate(text) if re.search(r"\b(rule|heads)\.backward\(", x))
    return "\n".join(x.strip() for x in text[first:last + 1])


def test_the_example():
    from paper_2607_19378_b200 import hyenand as hn
    B, H, Hk, D, dims = 2, 4, 2, 128, (64, 64)
    L, gen = 64 * 64, torch.Generator().manual_seed(61)
    n = lambda *s: torch.randn(s, generator=gen)
    t = dict(q=n(B, Hk * D, *dims).bfloat16(), k=n(B, Hk * D, *dims).bfloat16(), v=n(B, H * D, L).bfloat16(), dy=n(B, H * D, L).bfloat16(),
             g=-0.1 * torch.rand((B, H, L), generator=gen), beta=torch.rand((B, H, L), generator=gen), S0=0.3 * n(B, H, D, D), dS=0.3 * n(B, H, D, D),
             lengths=torch.tensor([130, 0], dtype=torch.int32))
    env = dict({k: v.cuda() for k, v in t.items()}, hn=hn, torch=torch, B=B, H=H, Hk=Hk, Hq=Hk)
    exec(lines(), env)
    torch.cuda.synchronize()
    q2, k2 = (env[x].cpu() for x in ("q2", "k2"))
    for x, y in ((t["q"], q2), (t["k"], k2)):
        assert oracle.rel_l2(y, oh.heads(x, Hk, dims, (32, 32), "l2")) <= 2.0 ** -8
    flat = lambda x: x.reshape(B, -1, L)
    ref = od.delta(flat(q2), flat(k2), t["v"], t["g"], t["beta"], "log", H, Hk, t["S0"], t["lengths"], t["dy"], t["dS"])
    for name, key in (("y", "y"), ("S", "s_end"), ("dq2", "dq"), ("dk2", "dk"), ("dv", "dv"), ("dg", "dg"), ("dbeta", "dbeta"), ("dS0", "ds0")):
        got = env[name].cpu()
        assert oracle.rel_l2(got, ref[key]) <= 7 * 2.0 ** -16 + (2.0 ** -8 if got.dtype == torch.bfloat16 else 0.0), name
