"""The operators together, as a layer uses them: norm, mixer (recurrence or causal long convolution), gated residual with dropout,
norm for the next layer; forward and gradients of the chain against torch autograd in 64 bits.

Tolerance: fp32 throughout; every operator is within a few 1e-6 of its exact value in the 2-norm (the convolution: 1e-5, its own
gate), and three of them follow one another in either direction: 4e-5."""
import pytest
import torch

import oracle
from oracle import block as ob

pytestmark = pytest.mark.gpu

EPS, P = 1e-6, 0.15


def rms(u, g):
    return u / torch.sqrt((u ** 2).mean(1, keepdim=True) + EPS) * g.view(1, -1, 1)


@pytest.mark.parametrize("mixer", ["recurrence", "convolution"])
def test_training_step(mixer):
    from paper_2607_19378_b200 import hyenand as hn
    B, C, L = 2, 48, 333
    gen = torch.Generator().manual_seed(31)
    n = lambda *s: torch.randn(s, generator=gen)
    x, z, q, v, f, do, dn = (n(B, C, L) for _ in range(7))
    h = n(C, L) * torch.exp(-torch.arange(L) / 30.0)
    g0, gp, sc, gn = 1 + 0.1 * n(C), 1 + 0.1 * n(C), 0.5 + 0.1 * n(C), 1 + 0.1 * n(C)
    rng = torch.tensor((77, 3), dtype=torch.int64, device="cuda")
    dev = {k: t.cuda() for k, t in dict(x=x, z=z, q=q, v=v, f=f, do=do, dn=dn, h=h, g0=g0, gp=gp, sc=sc, gn=gn).items()}

    # the library: the first norm is a block whose branch is nothing, then the mixer on the normed stream as k, then the block
    zero, nothing = torch.zeros_like(dev["x"]), torch.zeros(C, device="cuda")
    first = hn.Block((L,), B, C)
    _, k, st0 = first.forward(dev["x"], zero, scale=nothing, g_pre=dev["g0"], stats=True)
    if mixer == "recurrence":
        rec = hn.Recurrence(L, B, C, "sigmoid")
        m, _, marks = rec.forward(dev["q"], k, dev["v"], dev["f"], marks=True)
    else:
        plan = hn.Plan((L,), B, C, causal=True)
        m = plan.forward(dev["q"], k, dev["v"], dev["h"])
    blk = hn.Block((L,), B, C, gate="silu", p=P, site=4)
    w = dict(z=dev["z"], g_post=dev["gp"], scale=dev["sc"], g_pre=dev["gn"], rng=rng)
    r, nn, st = blk.forward(dev["x"], m, stats=True, **w)
    dx, dm, dz, dgp, dsc, dgn = blk.backward(dev["x"], m, st, dr=dev["do"], dn=dev["dn"], **w)
    if mixer == "recurrence":
        dq, dk, dv, dlast, _ = rec.backward(dev["q"], k, dev["v"], dev["f"], marks, dm)
    else:
        dq, dk, dv, dlast = hn.Backward((L,), B, C, mode="causal")(dev["q"], k, dev["v"], dev["h"], dm)
    dx0, _, _, _, _, dg0 = first.backward(dev["x"], zero, st0, scale=nothing, g_pre=dev["g0"], dr=dx, dn=dk)
    torch.cuda.synchronize()

    leaf = {k: t.double().requires_grad_(True) for k, t in dict(x=x, z=z, q=q, v=v, f=f, h=h, g0=g0, gp=gp, sc=sc, gn=gn).items()}
    kk = rms(leaf["x"], leaf["g0"])
    u = kk * leaf["v"]
    if mixer == "recurrence":
        a, s, rows = torch.sigmoid(leaf["f"]), torch.zeros(B, C, dtype=torch.float64), []
        for t in range(L):
            s = a[:, :, t] * s + u[:, :, t]
            rows.append(s)
        mm = leaf["q"] * torch.stack(rows, dim=-1)
    else:
        rows = [sum(leaf["h"][:, j] * u[:, :, t - j] for j in range(t + 1)) for t in range(L)]
        mm = leaf["q"] * torch.stack(rows, dim=-1)
    D = torch.from_numpy(ob.factor((B, C, L), P, (77, 3), 4))
    rr = leaf["x"] + leaf["sc"].view(1, C, 1) * (D * (torch.nn.functional.silu(leaf["z"]) * rms(mm, leaf["gp"])))
    out = rms(rr, leaf["gn"])
    names = ["x", "z", "q", "v", "f" if mixer == "recurrence" else "h", "g0", "gp", "sc", "gn"]
    want = dict(zip(names, torch.autograd.grad((rr * do).sum() + (out * dn).sum(), [leaf[k] for k in names])))
    got = dict(x=dx0, z=dz, q=dq, v=dv, g0=dg0, gp=dgp, sc=dsc, gn=dgn)
    got[names[4]] = dlast
    assert oracle.rel_l2(r.cpu(), rr.detach().numpy()) < 4e-5 and oracle.rel_l2(nn.cpu(), out.detach().numpy()) < 4e-5
    for k, t in got.items():
        assert oracle.rel_l2(t.cpu(), want[k].numpy()) < 4e-5, k
