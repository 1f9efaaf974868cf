"""CPU oracle of the gated linear recurrence -- TEST INFRASTRUCTURE ONLY.

    s_t = a_t s_{t-1} + k_t v_t,   y_t = q_t s_t,   a_t = g_t | exp(g_t) | 1 / (1 + exp(-g_t))

and its gradient, position by position in plain numpy float64.  Arrays [B, C, L]; s0, ds_end [B, C]; lengths: B integers or None.
Beside every result stands what bounds its rounding errors: the same sums over absolute values.
"""
from __future__ import annotations

import numpy as np

from . import to_f64


def decay(g: np.ndarray, kind: str):
    """a and da/dg"""
    if kind == "value":
        return g, np.ones_like(g)
    if kind == "log":
        a = np.exp(g)
        return a, a
    e = np.exp(-np.abs(g))
    a = np.where(g >= 0, 1.0, e) / (1.0 + e)
    return a, e / (1.0 + e) ** 2


def recurrence(q, k, v, g, kind, s0=None, lengths=None, dy=None, ds_end=None):
    """dict of y, s_end (and with dy: dq, dk, dv, dg, ds0), each with `<name>_abs`."""
    q, k, v, g = (to_f64(t) for t in (q, k, v, g))
    B, C, L = q.shape
    n = np.full(B, L) if lengths is None else np.clip(np.asarray(lengths), 0, L)
    live = np.arange(L)[None, None, :] < n[:, None, None]
    a, slope = decay(np.where(live, g, 0.0), kind)
    a = np.where(live, a, 1.0)
    u = np.where(live, np.where(live, k, 0.0) * np.where(live, v, 0.0), 0.0)
    q, k, v = (np.where(live, t, 0.0) for t in (q, k, v))
    state = np.zeros((B, C)) if s0 is None else to_f64(s0).copy()
    size = np.abs(state)
    s, sa, before, before_a = (np.empty_like(q) for _ in range(4))
    for t in range(L):
        before[:, :, t], before_a[:, :, t] = state, size
        state = a[:, :, t] * state + u[:, :, t]
        size = np.abs(a[:, :, t]) * size + np.abs(u[:, :, t])
        s[:, :, t], sa[:, :, t] = state, size
    out = {"y": q * s, "y_abs": np.abs(q) * sa, "s_end": state, "s_end_abs": size}
    if dy is None:
        return out
    dy = np.where(live, to_f64(dy), 0.0)
    mu = np.zeros((B, C)) if ds_end is None else to_f64(ds_end).copy()
    mua = np.abs(mu)
    lam, lama = np.empty_like(q), np.empty_like(q)
    for t in range(L - 1, -1, -1):
        lam[:, :, t] = q[:, :, t] * dy[:, :, t] + mu
        lama[:, :, t] = np.abs(q[:, :, t] * dy[:, :, t]) + mua
        mu, mua = a[:, :, t] * lam[:, :, t], np.abs(a[:, :, t]) * lama[:, :, t]
    out.update(dq=dy * s, dq_abs=np.abs(dy) * sa, dk=lam * v, dk_abs=lama * np.abs(v), dv=lam * k, dv_abs=lama * np.abs(k),
               dg=np.where(live, lam * before * slope, 0.0), dg_abs=np.where(live, lama * before_a * np.abs(slope), 0.0), ds0=mu, ds0_abs=mua)
    return out
