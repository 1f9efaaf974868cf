"""Heads whose squares lie beyond fp32 though their channels do not: they are normalised as any others, on grids of few tokens and of many,
and leave their neighbours as they are.

Bound: that of test_gpu_heads.py.  The scale by which such a head's channels are taken is a power of two and rounds nothing."""
import pytest
import torch

import oracle
from oracle import heads as oh
from test_gpu_heads import DTYPES, HALF, problem

pytestmark = pytest.mark.gpu


# lanes to a head: four rows of a warp, two warps, four, eight; single tokens; rows on 16 bytes and not
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("norm,eps", [("l2", 1e-6), ("rms", 1e-6), ("l2", 1e30)])
@pytest.mark.parametrize("T,D", [(1, 128), (7, 34), (8, 14), (20, 32), (33, 64), (72, 128), (65, 200), (136, 256)], ids=str)
def test_squares_beyond_fp32(T, D, norm, eps, dtype):
    from paper_2607_19378_b200 import hyenand as hn
    dt, axes = DTYPES[dtype], (D // 4,)
    t = problem((T,), axes, 2, 3, 2, D, dt, D + T)
    big = torch.zeros(T, dtype=torch.bool)
    big[::3] = True
    clean = {n: t[n].clone() for n in ("q", "k")}
    for n in ("q", "k"):                                     # every third token of one entry, at sizes up to the end of fp32
        x = t[n][1]
        x[:, big] = (x[:, big].float() / x[:, big].float().abs().max() * torch.logspace(19.5, 38.4, int(big.sum()))).to(dt)
    d = {n: None if v is None else v.cuda() for n, v in t.items()}
    op = hn.Heads((T,), 2, 3, 2, D, dt, norm, axes, eps=eps)
    w = dict(g_q=d["g_q"], g_k=d["g_k"])
    out = op.forward(d["q"], d["k"], **w)
    grads = op.backward(d["q"], d["k"], d["dq_out"], d["dk_out"], **w)
    small = op.forward(clean["q"].cuda(), clean["k"].cuda(), **w) + op.backward(clean["q"].cuda(), clean["k"].cuda(), d["dq_out"], d["dk_out"], **w)[:2]
    for i, (n, H) in enumerate((("q", 3), ("k", 2))):
        y, dx, dg = oh.heads(t[n], H, (T,), axes, norm, t["g_" + n], eps=eps, dout=t[f"d{n}_out"])
        exact = (D / 2 + 30) * 2.0 ** -24
        assert oracle.rel_l2(out[i].cpu(), y) <= HALF[dt] + exact, n
        assert oracle.rel_l2(out[i][1][:, big].cpu(), y[1][:, big.numpy()]) <= HALF[dt] + exact, n
        assert oracle.rel_l2(grads[i].cpu(), dx) <= HALF[dt] + 2 * exact, "d" + n
        # (their gradients are 1e-20 of the others'; from 1e37 on they and their roundings are below the smallest normal number)
        part = big & (t[n][1].float().abs().amax(0) < 1e30)
        assert oracle.rel_l2(grads[i][1][:, part].cpu(), dx[1][:, part.numpy()]) <= HALF[dt] + 2 * exact, "d" + n
        assert oracle.rel_l2(grads[2 + i].cpu(), dg) <= 1e-5, "dg_" + n
        for a, b in ((out[i], small[i]), (grads[i], small[2 + i])):
            assert torch.equal(a[0], b[0]) and torch.equal(a[1][:, ~big], b[1][:, ~big])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T,D", [(5, 64), (40, 64), (40, 16), (41, 130)], ids=str)
def test_infinities(T, D, dtype):
    """A channel without a finite value is NaN, the head's others are 0 beside it; other heads and tokens keep their bits."""
    from paper_2607_19378_b200 import hyenand as hn
    dt = DTYPES[dtype]
    t = problem((T,), (0,), 1, 2, 1, D, dt, 3)
    op = hn.Heads((T,), 1, 2, 1, D, dt, "l2")
    clean = op.forward(t["q"].cuda(), t["k"].cuda())[0].cpu()
    t["q"][0, D + 3, T // 2] = float("inf")
    y = op.forward(t["q"].cuda(), t["k"].cuda())[0].cpu()
    sick = y[0, D:, T // 2].float()
    assert bool(sick[3].isnan()) and float(torch.cat((sick[:3], sick[4:])).abs().max()) == 0.0
    y[0, D:, T // 2] = clean[0, D:, T // 2]
    assert torch.equal(y, clean)
