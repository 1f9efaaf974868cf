"""The delta rule over all that it allows: beta from 0 to 2, keys from unrelated to equal, decays to 1.

Near beta = 2 a token's key is reflected and not erased, and with keys that repeat the elimination of a chunk cancels what it is made of:
errors of the operands grow with that, in any arithmetic.  How far is taken from the formulas in 64 bits (chunks of 64, as the kernels have
them): every operand of every product is changed by a random part of what a product may be off by (test_gpu_delta.py: 2^-16 of bf16 tensors,
9 x 2^-23 of fp32 ones), and a result may move twice as far as the furthest of three such runs, or by the bound of test_gpu_delta.py."""
import numpy as np
import pytest
import torch

import oracle
from oracle import delta as od

NAMES = ("y", "s_end", "dq", "dk", "dv", "dg", "dbeta", "ds0")
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def chunked(t, change):
    """One value head to a head of keys, a "log" decay, [B H, ...] in 64 bits; `change` is applied to what enters a product."""
    B, H, L = t["beta"].shape
    wide = lambda x: oracle.to_f64(x).reshape(B * H, -1, L).transpose(0, 2, 1)
    q, k, v, dy = (wide(t[n]) for n in ("q", "k", "v", "dy"))
    g, beta = (oracle.to_f64(t[n]).reshape(B * H, L) for n in ("g", "beta"))
    mul = lambda a, b: change(a) @ change(b)
    T = lambda a: np.swapaxes(a, -1, -2)
    S = oracle.to_f64(t["s0"]).reshape(B * H, *t["s0"].shape[2:])
    kept, out = [], {n: np.zeros_like(x) for n, x in (("y", v), ("dq", q), ("dk", k), ("dv", v))}
    out.update(dg=np.zeros_like(g), dbeta=np.zeros_like(g))
    for t0 in range(0, L, 64):
        cut = slice(t0, min(t0 + 64, L))
        Q, K, V, G, be = q[:, cut], k[:, cut], v[:, cut], np.cumsum(g[:, cut], 1), beta[:, cut, None]
        n = Q.shape[1]
        low = np.tril(np.ones((n, n), bool))
        r = np.where(low, np.exp(np.where(low, G[:, :, None] - G[:, None, :], 0.0)), 0.0)
        gam, end = np.exp(G)[..., None], np.exp(G[:, -1:] - G)[..., None]
        KK = np.tril(r * (K @ T(K)), -1)
        A, P = np.linalg.inv(np.eye(n) + be * KK), r * (Q @ T(K))
        R = V - gam * mul(K, T(S))
        U = mul(A, be * R)
        kept.append((cut, S, Q, K, be, r, gam, end, KK, A, P, R, U))
        out["y"][:, cut] = gam * mul(Q, T(S)) + mul(P, U)
        S = gam[:, -1:] * S + mul(T(end * U), K)
    out["s_end"] = S
    D = oracle.to_f64(t["ds"]).reshape(S.shape)
    for cut, S, Q, K, be, r, gam, end, KK, A, P, R, U in reversed(kept):
        Y = dy[:, cut]
        dU = mul(T(P), Y) + end * mul(K, T(D))
        Z = mul(T(A), dU)
        F, E = np.tril(r * mul(Y, T(U))), -be * np.tril(r * mul(Z, T(U)), -1)
        of_q, of_k, of_end = gam * mul(Y, S), -be * gam * mul(Z, S), end * mul(U, D)
        out["dv"][:, cut], out["dq"][:, cut] = be * Z, of_q + mul(F, K)
        out["dk"][:, cut] = of_k + mul(E, K) + mul(T(F), Q) + mul(T(E), K) + of_end
        own = np.tril(r * mul(Z, T(U)), -1) * (K @ T(K))
        out["dbeta"][:, cut] = (Z * R).sum(2) - own.sum(2)
        M = np.tril(F, -1) * (Q @ T(K)) - be * own
        n = M.shape[1]
        across = np.stack([M[:, i:, :i].sum((1, 2)) for i in range(n)], 1)
        c, d = (Q * of_q + K * of_k).sum(2), (K * of_end).sum(2)
        w = gam[:, -1, 0] * (change(S) * D).sum((1, 2))
        out["dg"][:, cut] = across + np.cumsum(c[:, ::-1], 1)[:, ::-1] + np.cumsum(d, 1) - d + w[:, None]
        D = gam[:, -1:] * D + mul(T(gam * Y), Q) - mul(T(gam * be * Z), K)
    out["ds0"] = D
    return out


def problem(shape, dtype, beta, alike, g, seed=41):
    B, H, D, L = shape
    gen = torch.Generator().manual_seed(seed)
    n = lambda *s: torch.randn(s, generator=gen)
    unit = lambda x: x / x.norm(dim=2, keepdim=True)

    def heads():
        x = alike ** 0.5 * unit(n(B, H, D, 1)) + (1 - alike) ** 0.5 * unit(n(B, H, D, L))
        return unit(x).reshape(B, H * D, L).to(dtype)

    q, k = heads(), heads()
    return dict(q=q, k=k, v=n(B, H * D, L).to(dtype), dy=n(B, H * D, L).to(dtype), s0=0.3 * n(B, H, D, D), ds=0.3 * n(B, H, D, D),
                beta=torch.full((B, H, L), beta), g=torch.full((B, H, L), g), lengths=None)


def exact(t, H):
    ref = od.delta(t["q"], t["k"], t["v"], t["g"], t["beta"], "log", H, H, t["s0"], None, t["dy"], t["ds"])
    B, L = t["beta"].shape[0], t["beta"].shape[2]
    per = lambda n, x: x.reshape(B * H, -1, L).transpose(0, 2, 1) if n in ("y", "dq", "dk", "dv") else x.reshape((B * H,) + x.shape[2:])
    return {n: per(n, ref[n]) for n in NAMES}


def distance(a, b):
    rows = a.shape[0]
    return np.linalg.norm((a - b).reshape(rows, -1), axis=1) / (np.linalg.norm(b.reshape(rows, -1), axis=1) + 1e-30)


def test_the_chunks_are_the_rule():
    t = problem((2, 2, 12, 150), torch.float32, 1.7, 0.6, -0.05)
    got, ref = chunked(t, lambda x: x), exact(t, 2)
    assert all(distance(got[n], ref[n]).max() < 1e-11 for n in NAMES)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", [(1, 2, 64, 512), (1, 1, 128, 1100)], ids=str)
@pytest.mark.parametrize("beta,alike,g", [(1.0, 0.95, 0.0), (1.0, 1.0, -0.01), (1.5, 0.9, 0.0), (1.9, 0.9, -0.01), (2.0, 0.0, 0.0), (2.0, 0.95, 0.0), (2.0, 0.95, -0.1),
                                          (2.0, 1.0, 0.0)], ids=str)
def test_beta_and_keys(beta, alike, g, shape, dtype):
    from paper_2607_19378_b200 import hyenand as hn
    B, H, D, L = shape
    t = problem(shape, DTYPES[dtype], beta, alike, g)
    d = {n: None if x is None else x.cuda() for n, x in t.items()}
    op = hn.DeltaRule(L, B, H, D, dtype=DTYPES[dtype])
    x = [d[n] for n in ("q", "k", "v", "g", "beta")]
    y, s_end, marks = op.forward(*x, s0=d["s0"], marks=True)
    got = dict(zip(NAMES, (y, s_end) + op.backward(*x, marks, d["dy"], ds_end=d["ds"])))
    ref = exact(t, H)
    rng, size = np.random.default_rng(5), 2.0 ** -16 if dtype == "bf16" else 9 * 2.0 ** -23
    moved = [chunked(t, lambda a: a * (1 + size * rng.uniform(-1, 1, a.shape))) for _ in range(3)]
    for n in NAMES:
        a = oracle.to_f64(got[n].cpu())
        a = a.reshape(B * H, -1, L).transpose(0, 2, 1) if n in ("y", "dq", "dk", "dv") else a.reshape((B * H,) + a.shape[2:])
        bound = np.maximum(2 * np.max([distance(m[n], ref[n]) for m in moved], 0), 1e-5 if dtype == "f32" else 7 * 2.0 ** -16)
        bound += 2.0 ** -8 if got[n].dtype == torch.bfloat16 else 0.0
        err = distance(a, ref[n])
        assert np.all(err <= bound), (n, err, bound)
