"""Queries and keys as heads on the GPU against oracle/heads.py.

Bound, in the 2-norm of a tensor relative to it: a half step of the type (2^-24, 2^-8), and before it in fp32 a sum of D squares (D 2^-24, half
of it in the root), the root (2 x 2^-24), two products, and the angle's rotor: off by 2^-25 turns x 2 pi in the reduced angle, by 2^-23 in sine and
cosine and by 3 x 2^-24 in the product of two of them, 2 products and a sum more: (D / 2 + 30) 2^-24 in all; twice that for the gradients,
which form a second sum; the weights' gradients sum over all tokens in fp32, in chains of at most a few thousand: 2^-24 x sqrt of that
in the mean, 1e-5 held."""
import numpy as np
import pytest
import torch

import oracle
from oracle import heads as oh

pytestmark = pytest.mark.gpu

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}


def problem(dims, axes, B, Hq, Hk, D, dtype, seed, weights=True, positions=False, far=100000):
    g = torch.Generator().manual_seed(seed)
    n = lambda *s: torch.randn(s, generator=g)
    t = {"q": n(B, Hq * D, *dims).to(dtype), "k": n(B, Hk * D, *dims).to(dtype), "dq_out": n(B, Hq * D, *dims).to(dtype), "dk_out": n(B, Hk * D, *dims).to(dtype),
         "g_q": 1 + 0.2 * n(D) if weights else None, "g_k": 1 + 0.2 * n(D) if weights else None, "positions": None}
    if positions:
        t["positions"] = torch.randint(-far, far, (B, len(dims)) + dims, generator=g, dtype=torch.int32)
    return t


def check(dims, axes, B, Hq, Hk, D, dtype, norm, seed=1, weights=True, positions=False, base=10000.0, eps=1e-6):
    from paper_2607_19378_b200 import hyenand as hn
    dt = DTYPES[dtype]
    t = problem(dims, axes, B, Hq, Hk, D, dt, seed, weights, positions)
    d = {k: None if v is None else v.cuda() for k, v in t.items()}
    op = hn.Heads(dims, B, Hq, Hk, D, dt, norm, axes, base, eps)
    w = dict(g_q=d["g_q"], g_k=d["g_k"], positions=d["positions"])
    out = op.forward(d["q"], d["k"], **w)
    grads = op.backward(d["q"], d["k"], d["dq_out"], d["dk_out"], **w)
    torch.cuda.synchronize()
    for i, (name, H) in enumerate((("q", Hq), ("k", Hk))):
        y, dx, dg = oh.heads(t[name], H, dims, axes, norm, t["g_" + name], base, eps, t["positions"], t[f"d{name}_out"])
        exact = (D / 2 + 30) * 2.0 ** -24
        assert oracle.rel_l2(out[i].cpu(), y) <= HALF[dt] + exact, name
        assert oracle.rel_l2(grads[i].cpu(), dx) <= HALF[dt] + 2 * exact, "d" + name
        if weights:
            assert oracle.rel_l2(grads[2 + i].cpu(), dg) <= 1e-5, "dg_" + name
        else:
            assert grads[2 + i] is None


# head sizes on either side of what a lane's pairs hold; rows that start on 16 bytes and that do not; tiles that end inside a row of the
# grid and rows that end inside a tile; axes without pairs, channels without an axis
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("dims,axes,B,Hq,Hk,D,norm", [
    ((64,), (8,), 2, 2, 2, 16, "rms"), ((65,), (5,), 1, 3, 1, 12, "l2"), ((200,), (16,), 2, 2, 2, 32, "rms"), ((72,), (10,), 1, 2, 1, 34, "none"),
    ((16, 12), (16, 16), 2, 3, 3, 64, "l2"), ((9, 7), (3, 4), 3, 4, 2, 50, "rms"), ((128,), (64,), 1, 2, 2, 128, "l2"), ((40, 3), (20, 30), 1, 1, 1, 100, "rms"),
    ((5, 4, 8), (21, 21, 22), 1, 2, 1, 130, "rms"), ((33,), (100,), 1, 1, 1, 256, "l2"), ((3, 5, 7), (0, 2, 1), 2, 1, 2, 8, "none"), ((1,), (1,), 1, 1, 1, 2, "l2"),
    ((7,), (4,), 3, 5, 2, 64, "rms"), ((2, 2, 2), (1, 1, 1), 1, 1, 1, 6, "rms"), ((300, 1), (3, 3), 1, 9, 7, 24, "l2")], ids=str)
def test_shapes(dims, axes, B, Hq, Hk, D, norm, dtype):
    check(dims, axes, B, Hq, Hk, D, dtype, norm)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("dims,D", [((1,), 128), ((5,), 64), ((100,), 64), ((6, 5, 4), 48)])
def test_given_positions(dims, D, dtype):
    axes = (D // 2 // len(dims),) * len(dims)
    check(dims, axes, 3, 2, 1, D, dtype, "l2", positions=True)


# more tiles than CTAs, whose next rows are fetched a tile ahead, with positions of each batch entry's own; the largest table of a tile
@pytest.mark.parametrize("dims,axes,B,Hq,Hk,D,positions", [((44840,), (20,), 2, 1, 1, 40, True), ((44800,), (30,), 3, 2, 1, 62, False), ((24, 1), (32, 32), 5, 3, 2, 128, False),
                                                           ((24, 1), (32, 32), 5, 3, 2, 128, True)], ids=str)
def test_tiles_in_turn(dims, axes, B, Hq, Hk, D, positions):
    check(dims, axes, B, Hq, Hk, D, "bf16", "l2", positions=positions)


def test_no_weights_no_axes():
    check((50,), (0,), 2, 2, 1, 20, "f32", "rms", weights=False)


def test_far_positions():
    """Angles in 64 bits: positions of a billion and the end of a long row."""
    from paper_2607_19378_b200 import hyenand as hn
    t = problem((16,), (32,), 1, 1, 1, 64, torch.float32, 2, positions=True, far=1 << 30)
    y, _ = hn.Heads((16,), 1, 1, 1, 64, norm="none", axes=(32,)).forward(t["q"].cuda(), t["k"].cuda(), positions=t["positions"].cuda())
    assert oracle.rel_l2(y.cpu(), oh.heads(t["q"], 1, (16,), (32,), "none", positions=t["positions"])) <= 62 * 2.0 ** -24
    L = 262144
    q = torch.randn((1, 64, L), generator=torch.Generator().manual_seed(3))
    y, _ = hn.Heads((L,), 1, 1, 1, 64, norm="none", axes=(32,)).forward(q.cuda(), q.cuda())
    tail = torch.arange(L - 100, L).reshape(1, 1, 100)
    assert oracle.rel_l2(y[:, :, -100:].cpu(), oh.heads(q[:, :, -100:], 1, (100,), (32,), "none", positions=tail)) <= 62 * 2.0 ** -24


def test_zero_rows_and_large_ones():
    """A head of zeros has a norm of eps; squares near the end of fp32."""
    from paper_2607_19378_b200 import hyenand as hn
    x = torch.zeros(1, 16, 20)
    x[0, :, 5:] = torch.randn((16, 15), generator=torch.Generator().manual_seed(4))
    x[0, :, 10:] *= 1e17
    y, _ = hn.Heads((20,), 1, 1, 1, 16, norm="l2").forward(x.cuda(), x.cuda())
    assert float(y[0, :, :5].abs().max()) == 0.0
    assert oracle.rel_l2(y.cpu(), oh.heads(x, 1, (20,), (0,), "l2")) <= 40 * 2.0 ** -24


def test_in_place_on_another_stream_and_captured():
    from paper_2607_19378_b200 import hyenand as hn
    import os
    for dims in ((24, 31), (64, 8)):
        t = problem(dims, (6, 7), 2, 3, 2, 32, torch.bfloat16, 5)
        d = {k: None if v is None else v.cuda() for k, v in t.items()}
        op = hn.Heads(dims, 2, 3, 2, 32, torch.bfloat16, "rms", (6, 7))
        w = dict(g_q=d["g_q"], g_k=d["g_k"])
        calls = lambda: op.forward(d["q"], d["k"], **w) + op.backward(d["q"], d["k"], d["dq_out"], d["dk_out"], **w)
        want = calls()
        torch.cuda.synchronize()
        q, k = d["q"].clone(), d["k"].clone()
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        got = op.forward(q, k, **w, q_out=q, k_out=k, stream=side)
        side.synchronize()
        assert got[0].data_ptr() == q.data_ptr() and torch.equal(q, want[0]) and torch.equal(k, want[1])
        if os.environ.get("HYENAND_LIB") == "debug":
            continue                                          # that build synchronises in every call
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = calls()
        d["q"].mul_(2)
        graph.replay()
        torch.cuda.synchronize()
        d["q"].div_(2)
        assert torch.equal(out[1], want[1]) and not torch.equal(out[2], want[2])
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want))
