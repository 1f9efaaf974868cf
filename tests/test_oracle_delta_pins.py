"""Pins of the oracles of the delta rule and of heads (no GPU): worked values, torch autograd in 64 bits, central differences."""
import numpy as np
import pytest
import torch

from oracle import delta as od, heads as oh


def test_delta_by_hand():
    one = lambda *x: np.array(x, dtype=float).reshape(1, 1, -1)
    # one channel: S = 2, then 0.5 * 2 + 0.5 (4 - 0.5 * 2 * 1) 1 = 2.5, then 1.25 + 1 (3 - 1.25 * 2) 2 = 2.25
    r = od.delta(one(1, 2), one(1, 2), one(4, 3), one(np.log(0.5), np.log(0.5)), one(0.5, 1), "log", 1, 1, s0=np.full((1, 1, 1, 1), 2.0))
    assert np.allclose(r["y"], one(2.5, 4.5)) and np.allclose(r["s_end"], 2.25)


def test_delta_stores_and_replaces():
    """beta = 1 and orthonormal keys: the state gives back what was last written under a key."""
    rng = np.random.default_rng(0)
    D, Dv = 6, 4
    keys = np.linalg.qr(rng.standard_normal((D, D)))[0]
    order = [0, 1, 2, 3, 1, 0]
    k, v = keys[:, order][None], rng.standard_normal((1, Dv, 6))
    q = keys[:, [0, 0, 1, 2, 1, 3]][None]
    r = od.delta(q, k, v, None, np.ones((1, 1, 6)), "none", 1, 1)
    for t, last in enumerate([0, 0, 1, 2, 4, 3]):
        assert np.allclose(r["y"][0, :, t], v[0, :, last]), t


@pytest.mark.parametrize("kind", ["log", "sigmoid", "none"])
@pytest.mark.parametrize("lengths", [None, [5, 0, 3]])
def test_delta_gradients(kind, lengths):
    rng = np.random.default_rng(1)
    B, H, Hk, Dk, Dv, L = 3, 4, 2, 3, 2, 5
    n = [L] * B if lengths is None else lengths
    t = {s: torch.tensor(rng.standard_normal(shape), requires_grad=True) for s, shape in
         dict(q=(B, Hk * Dk, L), k=(B, Hk * Dk, L), v=(B, H * Dv, L), g=(B, H, L), beta=(B, H, L), s0=(B, H, Dv, Dk)).items()}
    dy, ds = torch.tensor(rng.standard_normal((B, H * Dv, L))), torch.tensor(rng.standard_normal((B, H, Dv, Dk)))
    a = {"log": torch.exp, "sigmoid": torch.sigmoid, "none": lambda x: torch.ones_like(x)}[kind](t["g"])
    total, ys, ends = 0.0, np.zeros((B, H * Dv, L)), np.zeros((B, H, Dv, Dk))
    for b in range(B):
        for h in range(H):
            S, cols = t["s0"][b, h], slice(h // 2 * Dk, (h // 2 + 1) * Dk)
            for i in range(n[b]):
                kt = t["k"][b, cols, i]
                S = a[b, h, i] * S
                S = S + torch.outer(t["beta"][b, h, i] * (t["v"][b, h * Dv:(h + 1) * Dv, i] - S @ kt), kt)
                y = S @ t["q"][b, cols, i]
                ys[b, h * Dv:(h + 1) * Dv, i] = y.detach()
                total = total + (y * dy[b, h * Dv:(h + 1) * Dv, i]).sum()
            ends[b, h] = S.detach()
            total = total + (S * ds[b, h]).sum()
    names = ["q", "k", "v", "beta", "s0"] + (["g"] if kind != "none" else [])
    grads = dict(zip(names, torch.autograd.grad(total, [t[s] for s in names])))
    r = od.delta(*(t[s].detach() for s in ("q", "k", "v", "g", "beta")), kind, H, Hk, t["s0"].detach(), lengths, dy, ds)
    assert np.allclose(r["y"], ys) and np.allclose(r["s_end"], ends)
    for s in names:
        assert np.allclose(r["d" + s], grads[s].numpy()), s


def test_delta_differences():
    rng = np.random.default_rng(2)
    B, H, D, L = 1, 1, 3, 4
    x = [rng.standard_normal(s) for s in ((B, D, L), (B, D, L), (B, D, L), (B, H, L), (B, H, L), (B, H, D, D))]
    dy, ds = rng.standard_normal((B, D, L)), rng.standard_normal((B, H, D, D))
    f = lambda y: (lambda r: (r["y"] * dy).sum() + (r["s_end"] * ds).sum())(od.delta(*y[:5], "sigmoid", H, H, y[5]))
    r = od.delta(*x[:5], "sigmoid", H, H, x[5], None, dy, ds)
    for i, name in enumerate(("dq", "dk", "dv", "dg", "dbeta", "ds0")):
        for at in np.ndindex(x[i].shape):
            up, down = [t.copy() for t in x], [t.copy() for t in x]
            up[i][at] += 1e-5
            down[i][at] -= 1e-5
            assert abs((f(up) - f(down)) / 2e-5 - r[name][at]) < 1e-7 * (1 + abs(r[name][at])) * 10, (name, at)


def test_heads_by_hand():
    x = np.array([3.0, 4.0]).reshape(1, 2, 1)
    assert np.allclose(oh.heads(x, 1, (1,), (1,), "l2", eps=0.0), [[[0.6], [0.8]]])
    at = np.array([2]).reshape(1, 1, 1)
    y = oh.heads(x, 1, (1,), (1,), "none", positions=at)[0, :, 0]
    assert np.allclose(y, [3 * np.cos(2) - 4 * np.sin(2), 3 * np.sin(2) + 4 * np.cos(2)])
    assert np.allclose(oh.heads(x, 1, (1,), (0,), "rms", eps=0.0)[0, :, 0], np.array([3, 4]) / np.sqrt(12.5))


def test_heads_depend_on_distance_only():
    """Turned queries and keys meet as their positions differ, axis by axis."""
    rng = np.random.default_rng(3)
    q, k = rng.standard_normal((1, 12, 1)), rng.standard_normal((1, 12, 1))
    at = lambda x, *p: oh.heads(x, 1, (1, 1), (2, 3), "none", positions=np.array(p).reshape(1, 2, 1))[0, :, 0]
    assert np.isclose(at(q, 5, 7) @ at(k, 2, 11), at(q, 3, 0) @ at(k, 0, 4))
    assert not np.isclose(at(q, 5, 7) @ at(k, 2, 11), at(q, 5, 7) @ at(k, 2, 12))


@pytest.mark.parametrize("norm", ["rms", "l2", "none"])
def test_heads_gradients(norm):
    rng = np.random.default_rng(4)
    B, H, D, dims, axes = 2, 3, 8, (3, 2), (1, 2)
    x, g = torch.tensor(rng.standard_normal((B, H * D) + dims), requires_grad=True), torch.tensor(rng.standard_normal(D), requires_grad=True)
    d = rng.standard_normal((B, H * D) + dims)
    z = x.reshape(B, H, D, -1)
    size = {"rms": lambda: torch.sqrt((z ** 2).mean(2, keepdim=True) + 1e-6), "l2": lambda: torch.sqrt((z ** 2).sum(2, keepdim=True) + 1e-6), "none": lambda: 1.0}[norm]()
    n = z / size * g.view(1, 1, D, 1)
    t = torch.tensor(oh.turns(dims, axes, D, 100.0))[:, None]
    lo, hi = n[:, :, :4], n[:, :, 4:]
    y = torch.cat([lo * torch.cos(t) - hi * torch.sin(t), lo * torch.sin(t) + hi * torch.cos(t)], dim=2).reshape(x.shape)
    dx, dg = torch.autograd.grad((y * torch.tensor(d)).sum(), (x, g))
    got = oh.heads(x.detach(), H, dims, axes, norm, g.detach(), 100.0, 1e-6, None, d)
    for a, b in zip(got, (y.detach(), dx, dg)):
        assert np.allclose(a, b.numpy())
