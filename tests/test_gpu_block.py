"""The residual block's operators and dropout on the GPU against oracle/block.py.

Bound of an element.  A rounding to the output type is at most eps(type) / 2 of the value.  Everything before it is fp32: a mean over
C channels is off by at most C/8 + 16 roundings of 2^-24 of its absolute terms, a normalised value by half that and 4 more, a gate by
8 (approximate exponential and quotient), the products and sums by 12 in all; dx and dm hold up to three such means behind one
another.  So |error| <= eps / 2 |ref| + K 2^-24 abs, K = 100 + C, with abs the same formula over absolute values.  The sums over all
tokens add at most one rounding per 32 tokens of the batch and 64 more.
"""
import numpy as np
import pytest
import torch

import oracle
from oracle import block as ob

pytestmark = pytest.mark.gpu

HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
EPS = 1e-6
RNG = (0x123456789ABCDEF, 5)


def guarded(like):
    n = like.numel()
    big = torch.full((n + 512,), 7.0, dtype=like.dtype, device="cuda")
    t = big[256:256 + n].view(like.shape)
    t.fill_(float("nan"))
    return big, t


def inputs(B, C, T, dtype, gate, post, scaled, pre, seed):
    g = torch.Generator().manual_seed(seed)
    n = lambda: torch.randn((B, C, T), generator=g).to(dtype)
    w = lambda s: (1.0 + 0.3 * torch.randn(C, generator=g)) * s
    t = {"x": n(), "m": n() * 3, "dr": n(), "dn": n(), "z": n() * 2 if gate != "none" else None}
    t.update(g_post=w(1.0) if post else None, scale=w(0.3) if scaled else None, g_pre=w(1.0) if pre else None)
    if not pre:
        t["dn"] = None
    return t


def run(t, B, C, T, dtype, gate, p, site=0, rng=RNG):
    """Forward and backward through the C ABI, every output between guard bands."""
    from paper_2607_19378_b200 import hyenand as hn
    d = {k: None if v is None else v.cuda() for k, v in t.items()}
    d["rng"] = torch.tensor(rng, dtype=torch.int64, device="cuda")
    code = {torch.float32: 0, torch.bfloat16: 1}[dtype]
    like = {"r": "x", "n": "x" if t["g_pre"] is not None else None, "dx": "x", "dm": "x", "dz": "z", "dg_post": "g_post", "dscale": "scale", "dg_pre": "g_pre"}
    bands = {k: guarded(d[v]) for k, v in like.items() if v and d[v] is not None}
    bands["stats"] = guarded(torch.empty(2 * B * T))
    bands["work"] = guarded(torch.empty(hn.hyenand_block_workspace_bytes(B, C, T, code) // 4))
    o = {k: None for k in like}
    o.update({k: b[1] for k, b in bands.items()})
    head = (B, C, T, code, d["x"], d["m"], d["z"], d["g_post"], d["scale"], d["g_pre"], EPS, {"none": 0, "sigmoid": 1, "silu": 2}[gate], p, d["rng"], site)
    hn.hyenand_block_forward(*head, o["r"], o["n"], o["stats"])
    for _ in range(2):                                       # the workspace keeps nothing that must be cleared
        hn.hyenand_block_backward(*head, o["stats"], d["dr"], d["dn"], o["dx"], o["dm"], o["dz"], o["dg_post"], o["dscale"], o["dg_pre"], o["work"])
    assert hn.hyenand_block_device_status() == 0, "a kernel gave up a bounded wait"
    for k, (big, x) in bands.items():
        assert bool((big[:256] == 7.0).all()) and bool((big[256 + x.numel():] == 7.0).all()), f"a kernel wrote outside {k}"
    return {k: v.cpu() for k, v in o.items() if v is not None and k not in ("stats", "work")}


def check(B, C, T, dtype, gate="silu", post=True, scaled=True, pre=True, p=0.0, seed=0, site=0):
    dt = DTYPES[dtype]
    t = inputs(B, C, T, dt, gate, post, scaled, pre, seed)
    got = run(t, B, C, T, dt, gate, p, site)
    D = ob.factor((B, C, T), p, RNG, site) if p else None
    ref = ob.block(t["x"], t["m"], t["z"], t["g_post"], t["scale"], t["g_pre"], EPS, gate, D, t["dr"], t["dn"])
    for k, v in got.items():
        half = HALF[v.dtype]
        K = 100 + C + (64 + B * T / 32 if v.dim() == 1 else 0)
        bound = half * np.abs(ref[k]) + K * 2.0 ** -24 * ref[k + "_abs"] * (1 + half) + 1e-37
        worst = np.max(np.abs(oracle.to_f64(v) - ref[k]) / bound)
        assert np.isfinite(worst) and worst <= 1.0, f"{k}: an element is off by {worst:.2f} x its bound"


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("gate", ["none", "sigmoid", "silu"])
@pytest.mark.parametrize("post,scaled,pre", [(True, True, True), (False, True, True), (True, False, False), (False, False, False), (True, True, False)])
def test_parts(gate, post, scaled, pre, dtype):
    check(3, 20, 37, dtype, gate, post, scaled, pre, seed=1)
    check(2, 24, 48, dtype, gate, post, scaled, pre, p=0.3, seed=2)


# tokens: one, odd, even, multiples of four and of eight, tiles that end inside; channels from one to thousands
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("B,C,T", [(1, 1, 1), (2, 3, 2), (3, 5, 4), (1, 7, 8), (2, 64, 210), (1, 33, 1023), (4, 100, 36), (2, 300, 31), (1, 768, 72), (2, 200, 1024),
                                   (1, 1000, 17), (1, 600, 35), (2, 700, 24), (1, 1030, 21), (1, 1500, 33), (1, 2048, 40), (1, 2100, 33), (1, 5000, 12), (70, 40, 9), (300, 17, 40), (2, 129, 66), (2, 90, 72), (1, 170, 80), (2, 380, 48), (1, 185, 45)], ids=str)
def test_sizes(B, C, T, dtype):
    check(B, C, T, dtype, p=0.2 if T % 3 else 0.0, seed=B + C + T, site=3)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_many_tokens(dtype):
    """More tiles than the backward has workspace slots."""
    check(2, 8, 40000, dtype, seed=4)
    check(3, 5, 20001, dtype, "sigmoid", seed=5, p=0.1)


def test_zero_tokens_and_saturated_gates():
    """A token of zeros in every channel, gates far out on both sides, dropped infinities."""
    B, C, T = 2, 30, 50
    t = inputs(B, C, T, torch.float32, "silu", True, True, True, 6)
    t["m"][:, :, 7] = 0.0
    t["x"][:, :, 7] = 0.0
    t["z"][0] = torch.sign(t["z"][0]) * 150.0
    got = run(t, B, C, T, torch.float32, "silu", 0.0)
    ref = ob.block(t["x"], t["m"], t["z"], t["g_post"], t["scale"], t["g_pre"], EPS, "silu", None, t["dr"], t["dn"])
    for k, v in got.items():
        K = 100 + C + 64
        assert np.all(np.abs(oracle.to_f64(v) - ref[k]) <= (K * ref[k + "_abs"] + np.abs(ref[k])) * 2.0 ** -24 + 1e-37), k
    t = inputs(1, 8, 16, torch.float32, "none", False, True, False, 7)
    gone = ~ob.keep(128, 0.5, *RNG).reshape(1, 8, 16)
    t["m"][torch.from_numpy(gone)] = float("inf")
    got = run(t, 1, 8, 16, torch.float32, "none", 0.5)
    assert bool(torch.isfinite(got["r"]).all()) and torch.equal(got["r"][torch.from_numpy(gone)], t["x"][torch.from_numpy(gone)])
    assert float(got["dm"][torch.from_numpy(gone)].abs().max()) == 0 and bool(torch.isfinite(got["dscale"]).all())


def test_one_gradient_given():
    from paper_2607_19378_b200 import hyenand as hn
    t = {k: v.cuda() for k, v in inputs(2, 40, 24, torch.float32, "silu", True, True, True, 8).items()}
    op = hn.Block((4, 6), 2, 40, gate="silu")
    shaped = {k: t[k].view(2, 40, 4, 6) for k in ("x", "m", "z", "dr", "dn")}
    w = dict(z=shaped["z"], g_post=t["g_post"], scale=t["scale"], g_pre=t["g_pre"])
    r, n, st = op.forward(shaped["x"], shaped["m"], stats=True, **w)
    zero = torch.zeros_like(shaped["dr"])
    for kw in (dict(dn=shaped["dn"]),):
        a = op.backward(shaped["x"], shaped["m"], st, dr=None, **w, **kw)
        b = op.backward(shaped["x"], shaped["m"], st, dr=zero, **w, **kw)
        assert all(torch.equal(u, v) for u, v in zip(a, b))
    with pytest.raises(hn.HyenaNDError):
        op.backward(shaped["x"], shaped["m"], st, dr=shaped["dr"], **w)       # dn belongs to g_pre
    with pytest.raises(ValueError):
        op.backward(shaped["x"], shaped["m"], st, dr=t["dr"], dn=shaped["dn"], **w)
    with pytest.raises(hn.HyenaNDError):
        hn.Block((4, 6), 2, 40, p=0.1).forward(shaped["x"], shaped["m"])      # no generator given


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n", [1, 7, 8, 9, 1000, 4099, 300001])
def test_dropout(n, dtype):
    """Every element: the product with the kept elements' factor, one rounding; in place; the block's mask is the same."""
    from paper_2607_19378_b200 import hyenand as hn
    dt = DTYPES[dtype]
    x = torch.randn(n, generator=torch.Generator().manual_seed(n)).to(dt)
    for p, site, rng in ((0.2, 0, (3, 1)), (0.5, 7, (-1, 2 ** 32 + 5)), (0.0, 1, (0, 0)), (0.99999, 2 ** 31 - 1, (2 ** 62 + 9, 1))):
        words = torch.tensor(rng, dtype=torch.int64, device="cuda")
        big, y = guarded(x.cuda())
        hn.Dropout(p, site)(x.cuda(), words, y=y)
        keep = torch.from_numpy(ob.keep(n, p, *rng, site))
        scale = torch.tensor(65536.0 / (65536 - ob.threshold(p)), dtype=torch.float32)
        want = torch.where(keep, x.float() * scale, torch.zeros(())).to(dt)
        assert torch.equal(y.cpu(), want)
        assert bool((big[:256] == 7.0).all()) and bool((big[256 + n:] == 7.0).all())
        z = x.cuda()
        assert hn.Dropout(p, site)(z, words, y=z) is z and torch.equal(z.cpu(), want)
    bad = x.clone()
    gone = ~torch.from_numpy(ob.keep(n, 0.5, 3, 1))
    bad[gone] = float("nan")
    out = hn.Dropout(0.5)(bad.cuda(), torch.tensor((3, 1), device="cuda"))
    assert bool(torch.isfinite(out).all())
    assert hn.Dropout(0.5)(torch.empty(0, device="cuda"), words).numel() == 0


def test_captured_dropout_draws_anew():
    """The generator's words are read on the device: a replayed graph drops what their new values say, in the block too."""
    from paper_2607_19378_b200 import hyenand as hn
    x = torch.randn((2, 16, 40), device="cuda")
    rng = torch.tensor((9, 0), dtype=torch.int64, device="cuda")
    drop, blk = hn.Dropout(0.25, site=2), hn.Block((40,), 2, 16, p=0.25, site=2)
    one = torch.ones(16, device="cuda")

    def step():
        y = drop(x, rng)
        r, _, st = blk.forward(x, x, scale=one, rng=rng, stats=True)
        return (y, r) + blk.backward(x, x, st, scale=one, rng=rng, dr=x)[:2]
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    masks = []
    for i in range(3):
        rng[1] = i
        graph.replay()
        torch.cuda.synchronize()
        keep = torch.from_numpy(ob.keep(x.numel(), 0.25, 9, i, 2)).view(x.shape).cuda()
        assert torch.equal(out[0] != 0, keep) and torch.equal(out[1] != x, keep) and torch.equal(out[3] != 0, keep)
        assert all(torch.equal(a, b) for a, b in zip(out, step()))
        masks.append(keep)
    assert not torch.equal(masks[0], masks[1]) and not torch.equal(masks[1], masks[2])


def test_two_backwards_at_once():
    """One handle on two streams and in two graphs: every call has its own workspace, the sums repeat bit for bit."""
    from paper_2607_19378_b200 import hyenand as hn
    op = hn.Block((50, 41), 3, 96, torch.bfloat16, gate="sigmoid")
    sets = []
    for s in (21, 22):
        t = {k: v.cuda() for k, v in inputs(3, 96, 2050, torch.bfloat16, "sigmoid", True, True, True, s).items()}
        sets.append({k: v.view(3, 96, 50, 41) if v.dim() == 3 else v for k, v in t.items()})

    def step(t, stream=None):
        w = dict(z=t["z"], g_post=t["g_post"], scale=t["scale"], g_pre=t["g_pre"], stream=stream)
        r, n, st = op.forward(t["x"], t["m"], stats=True, **w)
        return (r, n) + op.backward(t["x"], t["m"], st, dr=t["dr"], dn=t["dn"], **w)
    want = [step(t) for t in sets]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in sets]
    for _ in range(3):
        got = [step(t, s) for t, s in zip(sets, streams)]
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for g, w in zip(got, want) for a, b in zip(g, w))
    graphs, outs = [], []
    for t in sets:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            outs.append(step(t))
        graphs.append(graph)
    for _ in range(3):
        for graph, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for g, w in zip(outs, want) for a, b in zip(g, w))


def test_offsets_beyond_32_bits():
    """More than 2^31 elements: the last tokens against the oracle, dropout's counters at the end of the tensor."""
    from paper_2607_19378_b200 import hyenand as hn
    B, C, T = 1, 17, 130000008
    x = torch.zeros((B, C, T), dtype=torch.bfloat16, device="cuda")
    t = inputs(1, C, 40, torch.bfloat16, "none", True, True, True, 9)
    x[:, :, -40:] = t["x"].cuda()
    m = torch.zeros_like(x)
    m[:, :, -40:] = t["m"].cuda()
    w = {k: t[k].cuda() for k in ("g_post", "scale", "g_pre")}
    r, n = hn.Block((T,), B, C, torch.bfloat16).forward(x, m, **w)
    ref = ob.block(t["x"], t["m"], None, t["g_post"], t["scale"], t["g_pre"], EPS)
    for got, k in ((r, "r"), (n, "n")):
        err = np.abs(oracle.to_f64(got[:, :, -40:].cpu()) - ref[k])
        assert np.all(err <= HALF[torch.bfloat16] * np.abs(ref[k]) * 1.01 + (100 + C) * 2.0 ** -24 * ref[k + "_abs"]), k
        assert float(got[:, :, :100].abs().max()) == 0
    del r, n, m
    tail = x.numel() - x.numel() % 8 - 4096
    x.fill_(1.0)
    y = hn.Dropout(0.5, 1)(x, torch.tensor(RNG, device="cuda")).view(-1)
    k = ob.keep(x.numel() - tail, 0.5, *RNG, 1, first=tail)
    assert np.array_equal(y[tail:].cpu().float().numpy() != 0, k)
