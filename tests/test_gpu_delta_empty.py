"""Batch entries without tokens, or with next to none, among others, against the oracle: where value heads share keys, in segments, in CTAs that
take several chunks one after the other, at the first and last entry; states pass through them to the bit.

Bounds as in test_gpu_delta.py, but for dg and dbeta of entries of a few tokens.  Each of those is an inner product, <S_{t-1}, a_t dS_t> and
(dS_t k_t) . (v_t - a_t S_{t-1} k_t), and what its factors are off by grows no smaller where they happen to be next to orthogonal:
|<x + e, y + f> - <x, y>| <= |e| |y| + |x| |f|.  Over many tokens that evens out, over a few the bound is that of a result times the factors'
norms."""
import numpy as np
import pytest
import torch

import oracle
from oracle import delta as od
from test_gpu_delta import DTYPES, NAMES, bound, compare, inputs, run

pytestmark = pytest.mark.gpu
FEW = 8


def factors(t, ref, b, H, Hk):
    """Norms of the factors of dg and dbeta of entry b, [H, tokens]."""
    n = int(t["lengths"][b])
    cut = lambda i, to: [t[x][b:b + 1, :, i:to] for x in ("q", "k", "v", "g", "beta")] + ["log", H, Hk]
    norm = lambda x: np.linalg.norm(x.reshape(H, -1), axis=1)
    of_g, of_beta = np.zeros((H, n)), np.zeros((H, n))
    k = oracle.to_f64(t["k"])[b].reshape(Hk, -1, t["k"].shape[2]).repeat(H // Hk, axis=0)
    v, beta, a = oracle.to_f64(t["v"])[b].reshape(H, -1, t["v"].shape[2]), oracle.to_f64(t["beta"])[b], np.exp(oracle.to_f64(t["g"])[b])
    du = ref["dv"][b].reshape(v.shape) / beta[:, None]
    for i in range(n):
        before = oracle.to_f64(t["s0"])[b] if i == 0 else od.delta(*cut(0, i), t["s0"][b:b + 1])["s_end"][0]
        faded = od.delta(*cut(i, n), before[None], None, t["dy"][b:b + 1, :, i:n], t["ds"][b:b + 1])["ds0"]
        of_g[:, i] = norm(before) * norm(faded)
        e = v[:, :, i] - a[:, i, None] * np.einsum("hij,hj->hi", before, k[:, :, i])
        of_beta[:, i] = norm(du[:, :, i]) * norm(e)
    return {"dg": of_g, "dbeta": of_beta}


# several chunks a CTA of the gradients where B Hk chunks is above 148
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape,lengths", [
    ((40, 4, 4, 16, 16, 130), [0, 130, 1, 64, 65, 0, 0, 129, 128, 63] * 4), ((12, 6, 2, 32, 48, 520), [0, 520, 0, 0, 64, 300, 512, 513, 1, 0, 449, 0]),
    ((3, 1, 1, 64, 64, 1100), [0, 1100, 0]), ((4, 2, 1, 128, 40, 1056), [1056, 0, 5, 0]), ((4, 4, 2, 50, 97, 203), [0, 0, 203, 0]), ((2, 2, 1, 64, 64, 64), [0, 0]),
    ((1, 2, 2, 24, 24, 1100), [0])], ids=lambda x: str(x)[:24])
def test_entries_without_tokens(shape, lengths, dtype):
    B, H, Hk, Dk, Dv, L = shape
    t = inputs(*shape, DTYPES[dtype], "log", 51)
    t["lengths"] = torch.tensor(lengths, dtype=torch.int32)
    got = run(t, shape, DTYPES[dtype], "log")
    ref = od.delta(t["q"], t["k"], t["v"], t["g"], t["beta"], "log", H, Hk, t["s0"], t["lengths"], t["dy"], t["ds"])
    empty, few = t["lengths"] == 0, (t["lengths"] > 0) & (t["lengths"] < FEW)
    assert torch.equal(got["s_end"][empty], t["s0"][empty]) and torch.equal(got["ds0"][empty], t["ds"][empty])
    compare(got, ref, t, H, Hk, DTYPES[dtype], [n for n in NAMES if n not in ("dg", "dbeta")])
    part = {n: x[~few] for n, x in t.items()}
    compare({n: got[n][~few] for n in ("dg", "dbeta")}, {n: ref[n][(~few).numpy()] for n in ("dg", "dbeta")}, part, H, Hk, DTYPES[dtype], ["dg", "dbeta"])
    for b in few.nonzero()[:, 0].tolist():
        for n, size in factors(t, ref, b, H, Hk).items():
            off = np.abs(oracle.to_f64(got[n])[b] - ref[n][b])
            assert np.all(off[:, :lengths[b]] <= bound(torch.float32, DTYPES[dtype]) * size), (n, b)
            assert np.all(off[:, lengths[b]:] == 0), (n, b)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_what_lies_behind_a_length_against_the_oracle(dtype):
    """NaN and infinities behind the lengths, and lengths outside 0 .. L."""
    shape = B, H, Hk, Dk, Dv, L = 4, 2, 2, 32, 48, 144
    t = inputs(*shape, DTYPES[dtype], "log", 7)
    given, meant = torch.tensor([-3, 77, 1 << 30, 64], dtype=torch.int32), torch.tensor([0, 77, 144, 64], dtype=torch.int32)
    ref = od.delta(t["q"], t["k"], t["v"], t["g"], t["beta"], "log", H, Hk, t["s0"], meant, t["dy"], t["ds"])
    for b in range(B):
        for name, bad in (("q", "nan"), ("k", "inf"), ("v", "nan"), ("g", "inf"), ("beta", "nan"), ("dy", "-inf")):
            t[name][b, :, meant[b]:] = float(bad)
    got = run(dict(t, lengths=given), shape, DTYPES[dtype], "log")
    compare(got, ref, dict(t, lengths=meant), H, Hk, DTYPES[dtype], NAMES)
