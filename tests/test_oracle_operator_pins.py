"""Pins of the oracles of the recurrence, the residual block and dropout (no GPU): worked values, torch autograd in 64 bits, central
differences, and the published answers of the generator."""
import numpy as np
import pytest
import torch

from oracle import block as ob, recurrence as orec


def test_recurrence_by_hand():
    one = lambda *x: np.array(x, dtype=float).reshape(1, 1, -1)
    r = orec.recurrence(one(2, 1, -1), one(1, 3, 2), one(4, 1, 1), one(9, 0.5, -2), "value", s0=np.array([[0.25]]))
    # s: 9/4 + 4, then half of it + 3, then -2 times that + 2
    assert np.allclose(r["y"], one(2 * 6.25, 6.125, 10.25)) and np.allclose(r["s_end"], -10.25)
    r = orec.recurrence(one(2, 1, -1), one(1, 3, 2), one(4, 1, 1), one(9, 0.5, -2), "value", lengths=[2])
    assert np.allclose(r["y"], one(8, 5, 0)) and np.allclose(r["s_end"], 5)


@pytest.mark.parametrize("kind", ["value", "log", "sigmoid"])
@pytest.mark.parametrize("lengths", [None, [7, 0, 3]])
def test_recurrence_gradients(kind, lengths):
    rng = np.random.default_rng(1)
    B, C, L = 3, 2, 7
    q, k, v, g, dy = (torch.tensor(rng.standard_normal((B, C, L)), requires_grad=True) for _ in range(5))
    s0, ds = (torch.tensor(rng.standard_normal((B, C)), requires_grad=True) for _ in range(2))
    n = [L] * B if lengths is None else lengths
    a = {"value": lambda t: t, "log": torch.exp, "sigmoid": torch.sigmoid}[kind](g)
    rows, ends = [], []
    for b in range(B):
        s, ys = s0[b], []
        for t in range(n[b]):
            s = a[b, :, t] * s + k[b, :, t] * v[b, :, t]
            ys.append(q[b, :, t] * s)
        ys += [torch.zeros(C, dtype=torch.float64)] * (L - n[b])
        rows.append(torch.stack(ys, dim=-1))
        ends.append(s)
    y, end = torch.stack(rows), torch.stack(ends)
    grads = torch.autograd.grad((y * dy).sum() + (end * ds).sum(), (q, k, v, g, s0))
    r = orec.recurrence(*(t.detach() for t in (q, k, v, g)), kind, s0.detach(), lengths, dy.detach(), ds.detach())
    for name, want in zip(("y", "s_end", "dq", "dk", "dv", "dg", "ds0"), (y, end) + grads):
        assert np.allclose(r[name], want.detach().numpy(), atol=1e-12), name
        assert np.all(r[name + "_abs"] >= np.abs(r[name]) - 1e-12), name


def test_generator_published_answers():
    """Known answers published with the generator: zero counter and key, all ones, and digits of pi."""
    cases = [((0,) * 4, (0, 0), (0x6627e8d5, 0xe169c58d, 0xbc57ac4c, 0x9b00dbd8)),
             ((ob.M32,) * 4, (ob.M32, ob.M32), (0x408f276d, 0x41c83b0e, 0xa20bc7c6, 0x6d5451fd)),
             ((0x243f6a88, 0x85a308d3, 0x13198a2e, 0x03707344), (0xa4093822, 0x299f31d0), (0xd16cfe09, 0x94fdcceb, 0x5001e420, 0x24126ea1))]
    for counter, key, want in cases:
        assert tuple(int(w) for w in ob.philox4x32([np.array(c) for c in counter], key)) == want


def test_dropout_statistics():
    k = ob.keep(1 << 16, 0.25, seed=7, step=3)
    assert abs(k.mean() - 0.75) < 5 * np.sqrt(0.25 * 0.75 / k.size)
    assert (k != ob.keep(1 << 16, 0.25, seed=7, step=4)).any() and (k != ob.keep(1 << 16, 0.25, seed=7, step=3, site=1)).any()
    assert (ob.keep(160, 0.25, 7, 3)[80:] == ob.keep(80, 0.25, 7, 3, first=80)).all()
    assert ob.keep(64, 0.0, 7, 3).all() and ob.threshold(0.5) == 32768 and ob.threshold(0.999999) == 65535


@pytest.mark.parametrize("kind", ["none", "sigmoid", "silu"])
@pytest.mark.parametrize("post,scaled,pre", [(True, True, True), (False, True, True), (True, False, False)])
def test_block_gradients(kind, post, scaled, pre):
    rng = np.random.default_rng(2)
    B, C, T = 2, 5, 3
    t = lambda *s: torch.tensor(rng.standard_normal(s), requires_grad=True)
    x, m, z, dr, dn = (t(B, C, T) for _ in range(5))
    gp, sc, gn = t(C), t(C), t(C)
    D = (rng.random((B, C, T)) < 0.8) / 0.8
    rms = lambda u: u / torch.sqrt((u ** 2).mean(1, keepdim=True) + 1e-6)
    col = lambda u: u.view(1, C, 1)
    w = rms(m) * col(gp) if post else m
    if kind != "none":
        w = w * (torch.nn.functional.silu(z) if kind == "silu" else torch.sigmoid(z))
    r = x + (col(sc) if scaled else 1.0) * (torch.tensor(D) * w)
    loss = (r * dr).sum()
    want = {"r": r}
    if pre:
        n = rms(r) * col(gn)
        loss, want["n"] = loss + (n * dn).sum(), n
    names = ["dx", "dm"] + ["dz"] * (kind != "none") + ["dg_post"] * post + ["dscale"] * scaled + ["dg_pre"] * pre
    leaves = {"dx": x, "dm": m, "dz": z, "dg_post": gp, "dscale": sc, "dg_pre": gn}
    want.update(zip(names, torch.autograd.grad(loss, [leaves[k] for k in names])))
    got = ob.block(x.detach(), m.detach(), z.detach() if kind != "none" else None, gp.detach() if post else None, sc.detach() if scaled else None,
                   gn.detach() if pre else None, 1e-6, kind, D, dr.detach(), dn.detach() if pre else None)
    for name, val in want.items():
        assert np.allclose(got[name], val.detach().numpy(), atol=1e-12), name
        assert np.all(got[name + "_abs"] >= np.abs(got[name]) - 1e-12), name


def test_block_gradients_by_differences():
    """Central differences of the loss <r, dr> + <n, dn>: second-order error h^2 ~ 1e-10, rounding 1e-16 / h."""
    rng = np.random.default_rng(3)
    B, C, T, h = 1, 4, 2, 1e-5
    x, m, z, dr, dn = (rng.standard_normal((B, C, T)) for _ in range(5))
    gp, sc, gn = (rng.standard_normal(C) for _ in range(3))
    loss = lambda x, m, z: (lambda o: np.sum(o["r"] * dr) + np.sum(o["n"] * dn))(ob.block(x, m, z, gp, sc, gn, 1e-6, "silu"))
    got = ob.block(x, m, z, gp, sc, gn, 1e-6, "silu", None, dr, dn)
    for i, name in enumerate(("dx", "dm", "dz")):
        for idx in np.ndindex(B, C, T):
            args, lo = [x.copy(), m.copy(), z.copy()], None
            args[i][idx] += h
            hi = loss(*args)
            args[i][idx] -= 2 * h
            lo = loss(*args)
            assert abs((hi - lo) / (2 * h) - got[name][idx]) < 1e-7, (name, idx)
