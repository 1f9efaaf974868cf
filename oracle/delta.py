"""CPU oracle of the gated delta rule -- TEST INFRASTRUCTURE ONLY.

    u_t = beta_t (v_t - a_t S_{t-1} k_t),   S_t = a_t S_{t-1} + u_t k_t^T,   y_t = S_t q_t,   a_t = exp(g_t) | 1 / (1 + exp(-g_t)) | 1

and its gradient, token by token in plain numpy float64.  q, k [B, Hk D, L], v [B, H Dv, L], g, beta [B, H, L], states [B, H, Dv, Dk];
value head h goes with head h // (H // Hk) of queries and keys.  lengths: B integers or None.
"""
from __future__ import annotations

import numpy as np

from . import to_f64


def decay(g: np.ndarray, kind: str):
    """a and d a / d g"""
    if kind == "log":
        return np.exp(g), np.exp(g)
    e = np.exp(-np.abs(g))
    return np.where(g >= 0, 1.0, e) / (1.0 + e), e / (1.0 + e) ** 2


def delta(q, k, v, g, beta, kind, H, Hk, s0=None, lengths=None, dy=None, ds_end=None):
    """dict of y, s_end (and with dy: dq, dk, dv, dg, dbeta, ds0; dg is None for kind "none")."""
    q, k, v, beta = (to_f64(t) for t in (q, k, v, beta))
    B, L, share = q.shape[0], q.shape[2], H // Hk
    Dk, Dv = q.shape[1] // Hk, v.shape[1] // H
    a, slope = (np.ones_like(beta), None) if kind == "none" else decay(to_f64(g), kind)
    n = np.full(B, L) if lengths is None else np.clip(np.asarray(lengths), 0, L)
    start = np.zeros((B, H, Dv, Dk)) if s0 is None else to_f64(s0)
    out = {"y": np.zeros((B, H * Dv, L)), "s_end": start.copy()}
    if dy is not None:
        dy = to_f64(dy)
        out.update(dq=np.zeros(q.shape), dk=np.zeros(k.shape), dv=np.zeros(v.shape), dg=None if slope is None else np.zeros(beta.shape),
                   dbeta=np.zeros(beta.shape), ds0=np.zeros(start.shape) if ds_end is None else to_f64(ds_end).copy())
    for b in range(B):
        for h in range(H):
            rows, cols = slice(h * Dv, (h + 1) * Dv), slice(h // share * Dk, (h // share + 1) * Dk)
            Q, K, V = q[b, cols], k[b, cols], v[b, rows]
            S, before = start[b, h], []
            for t in range(n[b]):
                before.append(S)
                S = a[b, h, t] * S
                S = S + np.outer(beta[b, h, t] * (V[:, t] - S @ K[:, t]), K[:, t])
                out["y"][b, rows, t] = S @ Q[:, t]
            out["s_end"][b, h] = S
            if dy is None:
                continue
            D = out["ds0"][b, h].copy()
            for t in range(n[b] - 1, -1, -1):
                kt, qt, w = K[:, t], Q[:, t], dy[b, rows, t]
                faded = a[b, h, t] * before[t]
                e = V[:, t] - faded @ kt
                after = faded + np.outer(beta[b, h, t] * e, kt)
                out["dq"][b, cols, t] += after.T @ w
                D = D + np.outer(w, qt)
                du = D @ kt
                de = beta[b, h, t] * du
                out["dbeta"][b, h, t] = du @ e
                out["dv"][b, rows, t] = de
                out["dk"][b, cols, t] += D.T @ (beta[b, h, t] * e) - faded.T @ de
                D = D - np.outer(de, kt)
                if slope is not None:
                    out["dg"][b, h, t] = np.sum(D * before[t]) * slope[b, h, t]
                D = a[b, h, t] * D
            out["ds0"][b, h] = D
    return out
