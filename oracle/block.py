"""CPU oracle of a residual block's norms, gate, dropout and scale, and of dropout from counters -- TEST INFRASTRUCTURE ONLY.

    w = act(z) RMSNorm(m; g_post),   r = x + scale D w,   n = RMSNorm(r; g_pre)

in plain numpy float64 on [B, C, T], norms over the channels of a token; gradients by the chain rule, one factor at a time.  Beside
every result stands what bounds its rounding errors: the same sums over absolute values.
"""
from __future__ import annotations

import numpy as np

from . import to_f64

M32 = 0xFFFFFFFF


def philox4x32(counter, key, rounds: int = 10):
    """Salmon, Moraes, Dror, Shaw (SC 2011): four arrays of 32-bit words from four, key of two integers."""
    c = [np.asarray(w, dtype=np.uint64) for w in counter]
    k = [int(key[0]), int(key[1])]
    mask, sh = np.uint64(M32), np.uint64(32)
    for _ in range(rounds):
        p, r = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(r >> sh) ^ c[1] ^ np.uint64(k[0]), r & mask, (p >> sh) ^ c[3] ^ np.uint64(k[1]), p & mask]
        k = [(k[0] + 0x9E3779B9) & M32, (k[1] + 0xBB67AE85) & M32]
    return c


def threshold(p: float) -> int:
    return min(65535, int(np.floor(float(np.float32(p)) * 65536.0 + 0.5)))


def keep(n: int, p: float, seed: int, step: int, site: int = 0, first: int = 0) -> np.ndarray:
    """Which of the elements [first, first + n) of a tensor stay (first a multiple of 8)."""
    idx = np.arange(first // 8, (first + n + 7) // 8, dtype=np.uint64)
    words = philox4x32([idx & np.uint64(M32), idx >> np.uint64(32), np.full_like(idx, step & M32), np.full_like(idx, site & M32)],
                       (seed & M32, (seed >> 32) & M32))
    halves = np.stack([h for w in words for h in (w & np.uint64(0xFFFF), w >> np.uint64(16))], axis=-1).reshape(-1)[:n]
    return halves >= threshold(p)


def factor(shape, p, rng, site=0) -> np.ndarray:
    thr = threshold(p)
    return keep(int(np.prod(shape)), p, rng[0], rng[1], site).reshape(shape) * (65536.0 / (65536 - thr))


def gate(z, kind):
    """act(z), its slope, and a bound of the slope's terms"""
    e = np.exp(-np.abs(z))
    s = np.where(z >= 0, 1.0, e) / (1.0 + e)
    t = np.where(z >= 0, e, 1.0) / (1.0 + e)
    if kind == "silu":
        return z * s, s * (1.0 + z * t), s * (1.0 + np.abs(z) * t)
    return s, s * t, s * t


def block(x, m, z=None, g_post=None, scale=None, g_pre=None, eps=1e-6, kind="none", D=None, dr=None, dn=None):
    """dict of r, n (and with dr or dn: dx, dm, dz, dg_post, dscale, dg_pre), each with `<name>_abs`."""
    x, m = to_f64(x), to_f64(m)
    col = lambda t: np.ones((1, x.shape[1], 1)) if t is None else to_f64(t).reshape(1, -1, 1)
    gp, sc, gn = col(g_post), col(scale), col(g_pre)
    norm = lambda t: np.sqrt(np.mean(t * t, axis=1, keepdims=True) + eps)
    Nm = norm(m) if g_post is not None else 1.0
    mh = m / Nm
    act, slope, slope_a = (1.0, 0.0, 0.0) if z is None else gate(to_f64(z), kind)
    D = 1.0 if D is None else D
    w = act * mh * gp
    branch = sc * (D * w)
    r, ra = x + branch, np.abs(x) + np.abs(branch)
    Nr = norm(r)
    out = {"r": r, "r_abs": ra}
    if g_pre is not None:
        out.update(n=r / Nr * gn, n_abs=ra / Nr * np.abs(gn))
    if dr is None and dn is None:
        return out
    dr = np.zeros_like(x) if dr is None else to_f64(dr)
    d, da = dr, np.abs(dr)
    if dn is not None:
        dn = to_f64(dn)
        e = dn * gn
        proj, proj_a = np.mean(e * r, axis=1, keepdims=True), np.mean(np.abs(e) * ra, axis=1, keepdims=True)
        d = d + e / Nr - r * proj / Nr ** 3
        da = da + np.abs(e) / Nr + ra * proj_a / Nr ** 3
        out.update(dg_pre=np.sum(dn * r / Nr, axis=(0, 2)), dg_pre_abs=np.sum(np.abs(dn) * ra / Nr, axis=(0, 2)))
    dw, dwa = sc * D * d, np.abs(sc) * D * da
    out.update(dx=d, dx_abs=da, dscale=np.sum(d * D * w, axis=(0, 2)), dscale_abs=np.sum(da * D * np.abs(w), axis=(0, 2)))
    if z is not None:
        out.update(dz=dw * mh * gp * slope, dz_abs=dwa * np.abs(mh * gp) * slope_a)
    df, dfa = dw * act, dwa * np.abs(act)
    if g_post is None:
        out.update(dm=df, dm_abs=dfa)
        return out
    f, fa = df * gp, dfa * np.abs(gp)
    out.update(dg_post=np.sum(df * mh, axis=(0, 2)), dg_post_abs=np.sum(dfa * np.abs(mh), axis=(0, 2)),
               dm=(f - mh * np.mean(f * mh, axis=1, keepdims=True)) / Nm,
               dm_abs=(fa + np.abs(mh) * np.mean(fa * np.abs(mh), axis=1, keepdims=True)) / Nm)
    return out
