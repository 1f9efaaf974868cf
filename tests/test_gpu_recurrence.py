"""The gated linear recurrence on the GPU against oracle/recurrence.py.

Bound of an element.  A rounding to the output type is at most eps(type) / 2 of the value.  Everything before it is fp32, and every
term of a sum passes through a number of fp32 operations on its way to an element, counted in units of 2^-24: a decay from the
approximate exponential (4) and reciprocal (2) with the sum and product around them is off by at most 8, a step adds one more, so the
8 steps of a thread that a term starts in and the 8 of the one it ends in are 144 (16 of bf16 each: 288); 5 compositions between lanes
(5 each), one map a 256 positions or fewer (3 each), the products at the end (4).  So |error| <= eps / 2 |ref| + K 2^-24 abs, K = 176 +
L / 64 (bf16: 320 + L / 64), with abs the same sum over absolute values; a product of two such sums (dg) takes 2 K.
"""
import numpy as np
import pytest
import torch

import oracle
from oracle import recurrence as orec

pytestmark = pytest.mark.gpu

HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def inputs(B, C, L, dtype, decay, seed, ragged=False):
    g = torch.Generator().manual_seed(seed)
    t = {n: torch.randn((B, C, L), generator=g).to(dtype) for n in ("q", "k", "v", "dy")}
    raw = torch.randn((B, C, L), generator=g) + 6.0 * torch.rand((1, C, 1), generator=g)
    t["g"] = {"value": torch.sigmoid(raw), "log": -torch.exp(-raw), "sigmoid": raw}[decay].to(dtype)
    t["s0"], t["ds"] = torch.randn((B, C), generator=g), torch.randn((B, C), generator=g)
    t["lengths"] = torch.randint(0, L + 1, (B,), generator=g, dtype=torch.int32) if ragged else None
    return t


def guarded(like, dtype=None):
    n = like.numel()
    big = torch.full((n + 512,), 7.0, dtype=dtype or like.dtype, device="cuda")
    t = big[256:256 + n].view(like.shape)
    t.fill_(float("nan"))
    return big, t


def run(t, L, B, C, dtype, decay):
    """Forward and backward through the C ABI, every output between guard bands."""
    from paper_2607_19378_b200 import hyenand as hn
    d = {k: None if v is None else v.cuda() for k, v in t.items()}
    head = (B, C, L, {"value": 0, "log": 1, "sigmoid": 2}[decay], {torch.float32: 0, torch.bfloat16: 1}[dtype])
    bands = {n: guarded(d["q"]) for n in ("y", "dq", "dk", "dv", "dg")}
    bands.update({n: guarded(t["ds"]) for n in ("s_end", "ds0")})
    bands["marks"] = guarded(torch.empty(B, C, hn.hyenand_recurrence_marks(L)))
    bands["work"] = guarded(torch.empty(hn.hyenand_recurrence_workspace_bytes(B, C, L, head[4]) // 4))
    o = {n: b[1] for n, b in bands.items()}
    hn.hyenand_recurrence_forward(*head, d["q"], d["k"], d["v"], d["g"], d["s0"], d["lengths"], o["y"], o["s_end"], o["marks"], o["work"])
    hn.hyenand_recurrence_backward(*head, d["q"], d["k"], d["v"], d["g"], d["lengths"], o["marks"], d["dy"], d["ds"], o["dq"], o["dk"], o["dv"],
                                   o["dg"], o["ds0"], o["work"])
    assert hn.hyenand_recurrence_device_status() == 0, "a kernel gave up a bounded wait"
    for n, (big, x) in bands.items():
        assert bool((big[:256] == 7.0).all()) and bool((big[256 + x.numel():] == 7.0).all()), f"a kernel wrote outside {n}"
    return {n: x.cpu() for n, x in o.items()}


def compare(got, ref, L, names=("y", "s_end", "dq", "dk", "dv", "dg", "ds0")):
    K = (320 if got[names[0]].dtype == torch.bfloat16 else 176) + L / 64
    for n in names:
        half = HALF[got[n].dtype]
        bound = half * np.abs(ref[n]) + (2 * K if n == "dg" else K) * 2.0 ** -24 * ref[n + "_abs"] * (1 + half) + 1e-37
        err = np.abs(oracle.to_f64(got[n]) - ref[n])
        worst = np.max(err / bound)
        assert np.isfinite(worst) and worst <= 1.0, f"{n}: an element is off by {worst:.2f} x its bound"


def check(B, C, L, dtype, decay, seed, ragged=False):
    t = inputs(B, C, L, DTYPES[dtype], decay, seed, ragged)
    got = run(t, L, B, C, DTYPES[dtype], decay)
    ref = orec.recurrence(t["q"], t["k"], t["v"], t["g"], decay, t["s0"], t["lengths"], t["dy"], t["ds"])
    compare(got, ref, L)


# one position to several tiles; octets that rows share, tiles that end inside one, every number of lanes and of CTAs a row
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("decay", ["value", "log", "sigmoid"])
@pytest.mark.parametrize("L", [1, 2, 7, 8, 25, 26, 57, 58, 64, 65, 121, 122, 249, 256, 257, 505, 506, 1000, 1018, 1024, 1025, 2041, 2042, 2048, 3001, 4096, 4105])
def test_lengths(L, decay, dtype):
    check(2, 5, L, dtype, decay, seed=L, ragged=False)


@pytest.mark.parametrize("dtype,decay", [("f32", "log"), ("bf16", "sigmoid"), ("f32", "value")])
@pytest.mark.parametrize("B,C,L", [(7, 3, 13), (5, 4, 100), (6, 3, 700), (4, 3, 5003), (3, 200, 2050), (2, 300, 1029), (1, 160, 2500), (7, 2, 20011), (1, 199, 9000),
                                   (1, 205, 9001), (3, 150, 6000), (4, 160, 8200)], ids=str)
def test_padded_batches(B, C, L, dtype, decay):
    check(B, C, L, dtype, decay, seed=B * L, ragged=True)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_many_rows(dtype):
    """Rows that fill the GPU: one CTA a row."""
    check(2, 301, 1500, dtype, "sigmoid", seed=3)
    check(3, 700, 9, dtype, "log", seed=4)


def test_values_behind_an_entry_are_not_looked_at():
    """NaN and infinities behind the lengths reach nothing; y and the gradients are zero there; lengths of 0, of 1, beyond L."""
    B, C, L = 5, 3, 300
    t = inputs(B, C, L, torch.float32, "log", 5)
    t["lengths"] = torch.tensor([0, 1, 300, 10 ** 6, -4], dtype=torch.int32)
    clean = run(t, L, B, C, torch.float32, "log")
    for n, bad in zip(("q", "k", "v", "g", "dy"), (float("nan"), float("inf"), -float("inf"), float("nan"), float("inf"))):
        for b, m in enumerate([0, 1, 300, 300, 0]):
            t[n][b, :, m:] = bad
    got = run(t, L, B, C, torch.float32, "log")
    for n in clean:
        if n not in ("marks", "work"):
            assert torch.equal(clean[n], got[n]), n
    assert float(got["y"][0].abs().max()) == 0 and torch.equal(got["s_end"][0], t["s0"][0]) and torch.equal(got["ds0"][4], t["ds"][4])
    assert float(got["dg"][1, :, 1:].abs().max()) == 0


@pytest.mark.parametrize("dtype,L", [("f32", 20011), ("bf16", 40000)])
def test_entries_that_end_in_a_segment(dtype, L):
    """Few long rows, cut into segments: entries of no position, of one, of a part of the first segment, of all; NaN behind them."""
    lengths = [0, 1, 511, 512, 513, L - 1, L]
    t = inputs(len(lengths), 2, L, DTYPES[dtype], "sigmoid", 17)
    t["lengths"] = torch.tensor(lengths, dtype=torch.int32)
    ref = orec.recurrence(t["q"], t["k"], t["v"], t["g"], "sigmoid", t["s0"], t["lengths"], t["dy"], t["ds"])
    for n in ("q", "k", "v", "g", "dy"):
        for b, m in enumerate(lengths):
            t[n][b, :, m:] = float("nan")
    got = run(t, L, len(lengths), 2, DTYPES[dtype], "sigmoid")
    compare(got, ref, L)
    assert torch.equal(got["s_end"][0], t["s0"][0]) and torch.equal(got["ds0"][0], t["ds"][0])


@pytest.mark.parametrize("decay", ["value", "log", "sigmoid"])
def test_resets_and_extreme_gates(decay):
    """A decay of exactly zero cuts a row; gates of the type's lowest and highest values stay finite."""
    B, C, L = 2, 3, 400
    t = inputs(B, C, L, torch.float32, decay, 6)
    low = {"value": 0.0, "log": torch.finfo(torch.float32).min, "sigmoid": torch.finfo(torch.float32).min}[decay]
    high = {"value": 1.0, "log": 0.0, "sigmoid": torch.finfo(torch.float32).max}[decay]
    for at in (0, 5, 64, 255, 256, 390):
        t["g"][:, :, at] = low
    t["g"][:, 1, 100:200] = high
    t["g"][:, 2, :] = low
    if decay == "log":
        t["g"][:, 0, 300] = -float("inf")
    got = run(t, L, B, C, torch.float32, decay)
    ref = orec.recurrence(t["q"], t["k"], t["v"], t["g"], decay, t["s0"], None, t["dy"], t["ds"])
    compare(got, ref, L)


def test_negative_and_growing_decays():
    """Decays in [-1, 1], and above 1 over rows where nothing overflows (a product of 1.3 over 60 positions is 7e6; their roundings add
    up as those of any product, 60 more of 2^-24)."""
    for dtype in (torch.float32, torch.bfloat16):
        t = inputs(2, 3, 700, dtype, "value", 14)
        t["g"] = (2.0 * torch.rand(2, 3, 700, generator=torch.Generator().manual_seed(15)) - 1.0).to(dtype)
        compare(run(t, 700, 2, 3, dtype, "value"), orec.recurrence(t["q"], t["k"], t["v"], t["g"], "value", t["s0"], None, t["dy"], t["ds"]), 700)
        for decay, g in (("value", 1.3), ("log", 0.25)):
            t = inputs(2, 3, 60, dtype, decay, 16)
            t["g"].fill_(g)
            compare(run(t, 60, 2, 3, dtype, decay), orec.recurrence(t["q"], t["k"], t["v"], t["g"], decay, t["s0"], None, t["dy"], t["ds"]), 60 + 64 * 60)


@pytest.mark.parametrize("decay,g", [("log", -1e-6), ("log", -3e-5), ("sigmoid", 12.0), ("value", 1.0)])
def test_long_memories(decay, g):
    """A constant decay next to 1 over a long row: the rounding of each a_t, always to one side, must not add up."""
    B, C, L = 1, 2, 40000
    t = inputs(B, C, L, torch.float32, decay, 7)
    t["g"].fill_(g)
    got = run(t, L, B, C, torch.float32, decay)
    ref = orec.recurrence(t["q"], t["k"], t["v"], t["g"], decay, t["s0"], None, t["dy"], t["ds"])
    compare(got, ref, L)


def test_nan_spreads_to_later_positions_only():
    t = inputs(1, 2, 2000, torch.float32, "sigmoid", 8)
    t["k"][0, 0, 1234] = float("nan")
    got = run(t, 2000, 1, 2, torch.float32, "sigmoid")
    assert bool(torch.isfinite(got["y"][0, 0, :1234]).all()) and bool(torch.isnan(got["y"][0, 0, 1234:]).all()) and bool(torch.isfinite(got["y"][0, 1]).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("decay", ["value", "log", "sigmoid"])
def test_steps_follow_a_sequence(decay, dtype):
    """A prompt, then token by token in place: the oracle on the whole; entries that have ended keep their state."""
    from paper_2607_19378_b200 import hyenand as hn
    B, C, P, N = 3, 70, 33, 6
    t = inputs(B, C, P + N, DTYPES[dtype], decay, 9)
    d = {k: v.cuda() for k, v in t.items() if v is not None}
    part = lambda n, a, b: d[n][:, :, a:b].contiguous()
    y0, state = hn.Recurrence(P, B, C, decay, DTYPES[dtype]).forward(*(part(n, 0, P) for n in "qkvg"), s0=d["s0"])
    op, ys = hn.Recurrence(1, B, C, decay, DTYPES[dtype]), [y0]
    for i in range(P, P + N):
        ys.append(op.step(*(d[n][:, :, i].contiguous() for n in "qkvg"), state)[:, :, None])
    ref = orec.recurrence(t["q"], t["k"], t["v"], t["g"], decay, t["s0"])
    compare({"y": torch.cat(ys, dim=2).cpu(), "s_end": state.cpu()}, ref, P + N, ("y", "s_end"))
    before, new = state.clone(), torch.empty_like(state)
    y = op.step(*(d[n][:, :, 0].contiguous() for n in "qkvg"), state, new_state=new, active=torch.tensor([1, 0, 1], dtype=torch.int32, device="cuda"))
    assert torch.equal(state, before) and torch.equal(new[1], before[1]) and not torch.equal(new[0], before[0]) and float(y[1].abs().max()) == 0
    # a sequence of one position is the same step (its decay to within a few roundings: 1e-5 of a state is 168 of them)
    y1, end = op.forward(*(part(n, 0, 1) for n in "qkvg"), s0=state)
    y = op.step(*(d[n][:, :, 0].contiguous() for n in "qkvg"), state, new_state=new)
    assert torch.allclose(end, new, rtol=1e-5, atol=1e-5) and torch.allclose(y1[:, :, 0].float(), y.float(), rtol=2 * HALF[DTYPES[dtype]] + 1e-5, atol=1e-4)


def test_state_in_place_and_results_repeat():
    """s_end may be s0's buffer, ds0 ds_end's; two calls give the same bits; without s0, lengths and marks the same as with zeros."""
    from paper_2607_19378_b200 import hyenand as hn
    for B, C, L in ((2, 3, 50), (1, 4, 9000), (2, 300, 2100), (1, 3, 40001), (4, 29, 20000)):
        t = {k: v.cuda() for k, v in inputs(B, C, L, torch.bfloat16, "log", 10).items() if v is not None}
        op = hn.Recurrence(L, B, C, "log", torch.bfloat16)
        y, end, marks = op.forward(t["q"], t["k"], t["v"], t["g"], s0=t["s0"], marks=True)
        grads = op.backward(t["q"], t["k"], t["v"], t["g"], marks, t["dy"], ds_end=t["ds"])
        buf, y2 = t["s0"].clone(), torch.empty_like(y)
        work = torch.empty(hn.hyenand_recurrence_workspace_bytes(B, C, L, 1), dtype=torch.uint8, device="cuda")
        hn.hyenand_recurrence_forward(B, C, L, 1, 1, t["q"], t["k"], t["v"], t["g"], buf, None, y2, buf, None, work)
        dbuf, outs = t["ds"].clone(), [torch.empty_like(y) for _ in range(4)]
        hn.hyenand_recurrence_backward(B, C, L, 1, 1, t["q"], t["k"], t["v"], t["g"], None, marks, t["dy"], dbuf, *outs, dbuf, work)
        torch.cuda.synchronize()
        assert torch.equal(y, y2) and torch.equal(end, buf) and all(torch.equal(a, b) for a, b in zip(grads, outs + [dbuf]))
        zero, full = torch.zeros_like(t["s0"]), torch.full((B,), L, dtype=torch.int32, device="cuda")
        a, b = op.forward(t["q"], t["k"], t["v"], t["g"]), op.forward(t["q"], t["k"], t["v"], t["g"], s0=zero, lengths=full)
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


def test_captured_and_on_other_streams():
    """One handle in two graphs and on two streams at once: a call holds nothing that another could share."""
    from paper_2607_19378_b200 import hyenand as hn
    B, C, L = 2, 200, 3000
    op = hn.Recurrence(L, B, C, "sigmoid", torch.bfloat16)
    sets = [{k: v.cuda() for k, v in inputs(B, C, L, torch.bfloat16, "sigmoid", s).items() if v is not None} for s in (11, 12)]

    def step(t, stream=None):
        y, end, marks = op.forward(t["q"], t["k"], t["v"], t["g"], s0=t["s0"], marks=True, stream=stream)
        return (y, end) + op.backward(t["q"], t["k"], t["v"], t["g"], marks, t["dy"], ds_end=t["ds"], stream=stream)
    want = [step(t) for t in sets]
    torch.cuda.synchronize()
    graphs, outs = [], []
    for t in sets:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            outs.append(step(t))
        graphs.append(graph)
    streams = [torch.cuda.Stream() for _ in sets]
    for _ in range(3):
        for graph, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                graph.replay()
    torch.cuda.synchronize()
    for o, w in zip(outs, want):
        assert all(torch.equal(a, b) for a, b in zip(o, w))
    eager = [step(t, stream=s) for t, s in zip(sets, streams)]
    torch.cuda.synchronize()
    for o, w in zip(eager, want):
        assert all(torch.equal(a, b) for a, b in zip(o, w))
    sets[0]["q"].copy_(sets[1]["q"])
    graphs[0].replay()
    new = step(sets[0])
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(outs[0], new)) and not torch.equal(new[0], want[0][0])


def test_refusals():
    from paper_2607_19378_b200 import hyenand as hn
    op = hn.Recurrence(8, 2, 3, "log", torch.float32)
    x = torch.zeros((2, 3, 8), device="cuda")
    for bad in (x[:, :, :7], x.bfloat16(), x.permute(1, 0, 2).contiguous().permute(1, 0, 2), torch.zeros((2, 3, 16), device="cuda")[:, :, ::2], x.cpu()):
        with pytest.raises(ValueError):
            op.forward(x, x, bad, x)
    for kw in (dict(s0=x), dict(s0=x[:, :, 0].contiguous().double()), dict(lengths=torch.zeros(2, device="cuda", dtype=torch.int64)), dict(y=x[:1])):
        with pytest.raises(ValueError):
            op.forward(x, x, x, x, **kw)
    with pytest.raises(ValueError):
        op.backward(x, x, x, x, torch.zeros((2, 3, 2), device="cuda"), x)
    with pytest.raises(hn.HyenaNDError):
        op.forward(x, x, x, x, y=x)


@pytest.mark.parametrize("dtype", ["bf16"])
def test_offsets_beyond_32_bits(dtype):
    """More than 2^31 elements: the last rows against the oracle."""
    from paper_2607_19378_b200 import hyenand as hn
    B, C, L = 1, 16400, 131072 + 3
    small = inputs(1, 2, L, DTYPES[dtype], "sigmoid", 13)
    big = {}
    for n in ("q", "k", "v", "g", "dy"):
        big[n] = torch.zeros((B, C, L), dtype=DTYPES[dtype], device="cuda")
        big[n][:, -2:] = small[n].cuda()
    op = hn.Recurrence(L, B, C, "sigmoid", DTYPES[dtype])
    y, end, marks = op.forward(big["q"], big["k"], big["v"], big["g"], marks=True)
    got = {"y": y[:, -2:].cpu(), "s_end": end[:, -2:].cpu()}
    assert float(y[:, :5].abs().max()) == 0
    del y
    grads = op.backward(big["q"], big["k"], big["v"], big["g"], marks, big["dy"])
    torch.cuda.synchronize()
    got.update({n: x[:, -2:].cpu() for n, x in zip(("dq", "dk", "dv", "dg", "ds0"), grads)})
    ref = orec.recurrence(small["q"], small["k"], small["v"], small["g"], "sigmoid", None, None, small["dy"])
    compare(got, ref, L)
