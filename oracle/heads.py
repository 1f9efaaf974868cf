"""CPU oracle of queries and keys as heads (norm and rotation by grid positions) -- TEST INFRASTRUCTURE ONLY.

Plain numpy float64 on [B, H D, L_1..L_N], pairs of channels as complex numbers, the norm's gradient by the chain rule.
"""
from __future__ import annotations

import numpy as np

from . import to_f64


def turns(dims, axes, D, base, positions=None):
    """Angles of the D / 2 pairs, [1 or B, D / 2, T]; pairs without an axis stay at 0."""
    if positions is None:
        positions = np.stack(np.meshgrid(*(np.arange(n) for n in dims), indexing="ij"))[None]
    p = np.asarray(positions, dtype=np.float64).reshape(len(positions), len(dims), -1)
    out = np.zeros((p.shape[0], D // 2, p.shape[2]))
    row = 0
    for n, pairs in enumerate(axes):
        for j in range(pairs):
            out[:, row] = p[:, n] * float(base) ** (-j / pairs)
            row += 1
    return out


def heads(x, H, dims, axes, norm, g=None, base=10000.0, eps=1e-6, positions=None, dout=None):
    """(y, and with dout: dx, dg)"""
    x = to_f64(x)
    B, D = x.shape[0], x.shape[1] // H
    z = x.reshape(B, H, D, -1)
    g = np.ones((D, 1)) if g is None else to_f64(g).reshape(D, 1)
    unit = np.exp(1j * turns(dims, axes, D, base, positions))[:, None]
    turn = lambda t, by: (lambda c: np.concatenate([c.real, c.imag], axis=2))((t[:, :, :D // 2] + 1j * t[:, :, D // 2:]) * by)
    count = {"rms": D, "l2": 1, "none": 0}[norm]
    size = np.sqrt((z ** 2).sum(2, keepdims=True) / count + eps) if count else np.ones_like(z[:, :, :1])
    y = turn(z / size * g, unit).reshape(x.shape)
    if dout is None:
        return y
    d = turn(to_f64(dout).reshape(z.shape), np.conj(unit))
    dg = (d * z / size).sum((0, 1, 3))
    d = d * g
    dx = d / size
    if count:
        dx = dx - z * (z * d).sum(2, keepdims=True) / (count * size ** 3)
    return y, dx.reshape(x.shape), dg
