"""The gated delta rule on the GPU against oracle/delta.py.

Bound of a head's result in the 2-norm, relative to it.  A result comes out of a chain of at most seven products (k k^T, its
elimination, S k, A Z, u k^T, and one more each way for the gradients) of operands whose norms stay about the same for keys of norm 1.
Tensors of fp32 enter as three bf16 numbers (rest 2^-25, products left out 3 x 2^-25), and a sum is cut off at 2^-23 of itself by each of its
at most eight instructions at full size: 8 x 2^-23 + 2^-23 a product, seven of them 7.5e-6, held to 1e-5.  Tensors of bf16 enter as they
are, what is computed from them as two bf16 numbers (rest 2^-17, the product of two rests left out: 2^-18 at most): 2^-16 a product, seven
of them 1.07e-4 for results in fp32; results in bf16 are off by half a step, 2^-8 of the value, more."""
import threading

import numpy as np
import pytest
import torch

import oracle
from oracle import delta as od

pytestmark = pytest.mark.gpu

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
CODES = {"log": 1, "sigmoid": 2, "none": 3}


def inputs(B, H, Hk, Dk, Dv, L, dtype, decay, seed, ragged=False):
    g = torch.Generator().manual_seed(seed)
    n = lambda *s: torch.randn(s, generator=g)

    def unit():
        x = n(B, Hk, Dk, L)
        return (x / x.norm(dim=2, keepdim=True).clamp_min(1e-6)).reshape(B, Hk * Dk, L).to(dtype)

    t = dict(q=unit(), k=unit(), v=n(B, H * Dv, L).to(dtype), beta=torch.sigmoid(n(B, H, L)), s0=0.3 * n(B, H, Dv, Dk), dy=n(B, H * Dv, L).to(dtype),
             ds=0.3 * n(B, H, Dv, Dk))
    t["g"] = {"log": -0.3 * torch.exp(n(B, H, L)), "sigmoid": 2 + 2 * n(B, H, L), "none": None}[decay]
    t["lengths"] = torch.randint(0, L + 1, (B,), generator=g, dtype=torch.int32) if ragged else None
    return t


def bound(result, dtype):
    exact = 1e-5 if dtype == torch.float32 else 7 * 2.0 ** -16
    return exact + (2.0 ** -8 if result == torch.bfloat16 else 0.0)


def compare(got, ref, t, H, Hk, dtype, names):
    for name in names:
        heads = Hk if name in ("dq", "dk") else H
        a, b = oracle.to_f64(got[name]), ref[name]
        a, b = a.reshape(a.shape[0], heads, -1), b.reshape(b.shape[0], heads, -1)
        size, err = np.linalg.norm(b, axis=2), np.linalg.norm(a - b, axis=2)
        assert np.all(np.isfinite(a)), name
        worst = np.max(err / (bound(got[name].dtype, dtype) * size + 1e-30))
        assert worst <= 1.0, f"{name}: a head is off by {worst:.2f} x its bound"
    if t["lengths"] is not None:
        dead = torch.arange(t["q"].shape[2])[None, :] >= t["lengths"][:, None]
        for name in set(names) & {"y", "dq", "dk", "dv", "dg", "dbeta"}:
            assert float(got[name].float().abs().sum(1)[dead].sum()) == 0.0, f"{name} behind a length"


def guarded(shape, dtype):
    n = int(np.prod(shape))
    big = torch.full((n + 512,), 7.0, dtype=dtype, device="cuda")
    x = big[256:256 + n].view(shape)
    x.fill_(float("nan"))
    return big, x


def run(t, shape, dtype, decay):
    """Forward and backward through the C ABI, every output and workspace between guard bands."""
    from paper_2607_19378_b200 import hyenand as hn
    B, H, Hk, Dk, Dv, L = shape
    d = {k: None if v is None else v.cuda() for k, v in t.items()}
    code = {torch.float32: 0, torch.bfloat16: 1}[dtype]
    head = (B, H, Hk, L, Dk, Dv, CODES[decay], code)
    bands = {n: guarded(t[s].shape, t[s].dtype) for n, s in dict(y="v", dq="q", dk="k", dv="v", dbeta="beta", s_end="s0", ds0="s0").items()}
    if decay != "none":
        bands["dg"] = guarded(t["g"].shape, torch.float32)
    bands["marks"] = guarded((B, H, hn.hyenand_delta_marks(L, Dk, Dv)), torch.float32)
    for n, back in (("work", 0), ("work_back", 1)):
        bands[n] = guarded((hn.hyenand_delta_workspace_bytes(B, H, Hk, L, Dk, Dv, code, back) // 4,), torch.float32)
    o = {n: b[1] for n, b in bands.items()}
    hn.hyenand_delta_forward(*head, d["q"], d["k"], d["v"], d["g"], d["beta"], d["s0"], d["lengths"], o["y"], o["s_end"], o["marks"], o["work"])
    hn.hyenand_delta_backward(*head, d["q"], d["k"], d["v"], d["g"], d["beta"], d["lengths"], o["marks"], d["dy"], d["ds"], o["dq"], o["dk"], o["dv"],
                              o.get("dg"), o["dbeta"], o["ds0"], o["work_back"])
    assert hn.hyenand_delta_device_status() == 0, "a kernel gave up a bounded wait"
    for n, (big, x) in bands.items():
        assert bool((big[:256] == 7.0).all()) and bool((big[256 + x.numel():] == 7.0).all()), f"a kernel wrote outside {n}"
    return {n: x.cpu() for n, x in o.items()}


NAMES = ("y", "s_end", "dq", "dk", "dv", "dg", "dbeta", "ds0")


def check(shape, dtype, decay, seed, ragged=False):
    B, H, Hk, Dk, Dv, L = shape
    t = inputs(*shape, DTYPES[dtype], decay, seed, ragged)
    got = run(t, shape, DTYPES[dtype], decay)
    ref = od.delta(t["q"], t["k"], t["v"], t["g"], t["beta"], decay, H, Hk, t["s0"], t["lengths"], t["dy"], t["ds"])
    compare(got, ref, t, H, Hk, DTYPES[dtype], [n for n in NAMES if n in got])


# one token to several chunks, ends inside a chunk and on its border; rows that are and are not multiples of 16 bytes; head sizes on
# either side of what a tile holds, values wider and narrower than keys; shared queries and keys
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape,decay,ragged", [
    ((1, 1, 1, 128, 128, 64), "none", False), ((2, 3, 3, 64, 64, 65), "log", False), ((2, 4, 2, 50, 97, 200), "sigmoid", True), ((3, 2, 1, 17, 5, 1), "log", False),
    ((1, 2, 2, 128, 64, 127), "sigmoid", False), ((2, 1, 1, 64, 128, 63), "none", True), ((1, 3, 1, 33, 64, 136), "log", True), ((4, 2, 2, 1, 1, 70), "log", True),
    ((2, 6, 3, 72, 72, 192), "log", True), ((1, 1, 1, 65, 66, 128), "sigmoid", False), ((5, 1, 1, 16, 16, 8), "none", True)], ids=str)
def test_shapes(shape, decay, ragged, dtype):
    check(shape, dtype, decay, 3, ragged)


# few heads and many chunks: cut into segments, the last of them short, entries that end in the first
@pytest.mark.parametrize("shape,dtype,decay,ragged", [((1, 1, 1, 64, 64, 1100), "bf16", "log", False), ((2, 2, 1, 128, 40, 1050), "f32", "sigmoid", True),
                                                      ((3, 1, 1, 24, 100, 1096), "bf16", "none", True), ((1, 3, 3, 128, 128, 1024), "bf16", "log", False)], ids=str)
def test_segments(shape, dtype, decay, ragged):
    check(shape, dtype, decay, 4, ragged)


# rows that tensor copies read but for the last chunk, which ends inside: its threads have passed over the chunks before (every stage, early and late)
@pytest.mark.parametrize("D", [64, 128])
def test_ragged_rows_of_many_chunks(D):
    shape = B, H, Hk, Dk, Dv, L = 10, 2, 1, D, D, 960
    t = inputs(*shape, torch.bfloat16, "log", 12)
    t["lengths"] = torch.tensor([900, 540, 300, 700, 959, 385, 449, 520, 960, 600], dtype=torch.int32)
    got = run(t, shape, torch.bfloat16, "log")
    ref = od.delta(t["q"], t["k"], t["v"], t["g"], t["beta"], "log", H, Hk, t["s0"], t["lengths"], t["dy"], t["ds"])
    compare(got, ref, t, H, Hk, torch.bfloat16, [n for n in NAMES if n in got])


# what one entry and one head hold reaches no other, though they share CTAs, shared and tensor memory one after the other
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("Dk,Dv,L", [(50, 41, 136), (40, 97, 130)])
def test_a_nan_stays_with_its_head(Dk, Dv, L, dtype):
    shape = B, H, Hk, Dk, Dv, L = 12, 12, 12, Dk, Dv, L
    t = inputs(*shape, DTYPES[dtype], "log", 13)
    sick = torch.zeros(B, H, dtype=torch.bool)
    sick[::3, ::2] = True
    clean = {k: None if v is None else v.clone() for k, v in t.items()}
    for name in ("q", "k", "v", "dy"):
        rows = t[name].view(B, H, -1, L)
        rows[sick] = float("nan") if name in ("q", "v") else float("inf")
    t["s0"][sick] = float("nan")
    got = run(t, shape, DTYPES[dtype], "log")
    ref = od.delta(clean["q"], clean["k"], clean["v"], clean["g"], clean["beta"], "log", H, Hk, clean["s0"], None, clean["dy"], clean["ds"])
    for n in NAMES:
        a, b = got[n].reshape(B * H, -1)[~sick.flatten()], torch.from_numpy(np.ascontiguousarray(ref[n])).reshape(B * H, -1)[~sick.flatten()]
        compare({n: a[None].reshape(1, len(a), -1)}, {n: b.numpy()[None]}, dict(clean, lengths=None), len(a), len(a), DTYPES[dtype], [n])


# more heads than SMs, and a batch entry without tokens among them
def test_many_heads():
    check((40, 4, 4, 16, 16, 130), "bf16", "log", 5, True)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_without_states_and_without_gradients_of_them(dtype):
    from paper_2607_19378_b200 import hyenand as hn
    shape = B, H, Hk, Dk, Dv, L = 2, 2, 1, 40, 24, 100
    t = inputs(*shape, DTYPES[dtype], "log", 6)
    d = {k: None if v is None else v.cuda() for k, v in t.items()}
    op = hn.DeltaRule(L, B, H, Dk, Dv, Hk, "log", DTYPES[dtype])
    y, s_end, marks = op.forward(d["q"], d["k"], d["v"], d["g"], d["beta"], marks=True)
    grads = op.backward(d["q"], d["k"], d["v"], d["g"], d["beta"], marks, d["dy"])
    got = {n: x.cpu() for n, x in zip(("y", "s_end", "dq", "dk", "dv", "dg", "dbeta", "ds0"), (y, s_end) + grads)}
    ref = od.delta(t["q"], t["k"], t["v"], t["g"], t["beta"], "log", H, Hk, None, None, t["dy"])
    compare(got, ref, t, H, Hk, DTYPES[dtype], NAMES)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_what_lies_behind_a_length_is_not_looked_at(dtype):
    shape = B, H, Hk, Dk, Dv, L = 4, 2, 2, 32, 48, 144
    t = inputs(*shape, DTYPES[dtype], "log", 7)
    t["lengths"] = torch.tensor([0, 77, 144, 64], dtype=torch.int32)
    clean = run(t, shape, DTYPES[dtype], "log")
    for b in range(B):
        for name in ("q", "k", "v", "g", "beta", "dy"):
            t[name][b, :, t["lengths"][b]:] = float("nan")
    t["lengths"] = torch.tensor([-3, 77, 1 << 30, 64], dtype=torch.int32)        # values outside count as the nearer end
    got = run(t, shape, DTYPES[dtype], "log")
    for name in NAMES:
        assert torch.equal(got[name], clean[name]), name


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_decays_that_forget_everything(dtype):
    shape = B, H, Hk, Dk, Dv, L = 1, 2, 2, 64, 64, 200
    t = inputs(*shape, DTYPES[dtype], "log", 8)
    t["g"][0, 0, [0, 70, 71, 130]] = torch.tensor([-float("inf"), -1e30, -200.0, -5000.0])
    got = run(t, shape, DTYPES[dtype], "log")
    t["g"].clamp_(min=-1e4)                                   # (exp of either is 0 in 64 bits too; the oracle's -inf would meet 0)
    ref = od.delta(t["q"], t["k"], t["v"], t["g"], t["beta"], "log", H, Hk, t["s0"], None, t["dy"], t["ds"])
    compare(got, ref, t, H, Hk, DTYPES[dtype], NAMES)
    assert float(got["ds0"][0, 0].abs().max()) == 0.0


def test_nothing_written_leaves_the_state():
    from paper_2607_19378_b200 import hyenand as hn
    shape = B, H, Hk, Dk, Dv, L = 2, 2, 2, 64, 32, 130
    t = inputs(*shape, torch.bfloat16, "none", 9)
    t["beta"].zero_()
    got = run(t, shape, torch.bfloat16, "none")
    ref = od.delta(t["q"], t["k"], t["v"], None, t["beta"], "none", H, Hk, t["s0"], None, t["dy"], t["ds"])
    assert torch.equal(got["s_end"], t["s0"])
    compare(got, ref, t, H, Hk, torch.bfloat16, ["y", "dq", "dbeta", "ds0"])
    assert float(got["dv"].float().abs().max()) == 0.0


def test_a_nan_stays_in_its_head_and_in_front_of_it_nothing():
    shape = B, H, Hk, Dk, Dv, L = 1, 3, 3, 64, 64, 300
    t = inputs(*shape, torch.bfloat16, "log", 10)
    clean = run(t, shape, torch.bfloat16, "log")
    t["v"][0, 64 + 5, 150] = float("nan")
    got = run(t, shape, torch.bfloat16, "log")
    y, c = got["y"].view(1, 3, 64, L), clean["y"].view(1, 3, 64, L)
    assert torch.equal(y[:, [0, 2]], c[:, [0, 2]]) and torch.equal(y[:, 1, :, :128], c[:, 1, :, :128])
    assert bool(torch.isnan(y[0, 1, 5, 150:]).all())


def test_states_in_their_own_buffers_and_other_streams():
    from paper_2607_19378_b200 import hyenand as hn
    shape = B, H, Hk, Dk, Dv, L = 2, 2, 2, 64, 64, 264
    t = {k: None if v is None else v.cuda() for k, v in inputs(*shape, torch.bfloat16, "log", 11).items()}
    op = hn.DeltaRule(L, B, H, Dk, Dv, Hk, "log", torch.bfloat16)
    x = (t["q"], t["k"], t["v"], t["g"], t["beta"])
    y, s_end, marks = op.forward(*x, s0=t["s0"], marks=True)
    grads = op.backward(*x, marks, t["dy"], ds_end=t["ds"])
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    y2, s2, marks2 = op.forward(*x, s0=t["s0"], marks=True, stream=side)
    grads2 = op.backward(*x, marks2, t["dy"], ds_end=t["ds"], stream=side.cuda_stream)
    side.synchronize()
    assert torch.equal(y, y2) and torch.equal(s_end, s2) and all(torch.equal(a, b) for a, b in zip(grads, grads2))
    # through the C ABI, s_end over s0 and ds0 over ds_end
    state, gradient, mk = t["s0"].clone(), t["ds"].clone(), torch.empty_like(marks)
    work = torch.empty(hn.hyenand_delta_workspace_bytes(B, H, Hk, L, Dk, Dv, 1, 1), dtype=torch.uint8, device="cuda")
    o = [torch.empty_like(a) for a in grads[:5]]
    hn.hyenand_delta_forward(B, H, Hk, L, Dk, Dv, 1, 1, *x, state, None, y2, state, mk, work)
    hn.hyenand_delta_backward(B, H, Hk, L, Dk, Dv, 1, 1, *x, None, mk, t["dy"], gradient, *o, gradient, work)
    torch.cuda.synchronize()
    assert torch.equal(y, y2) and torch.equal(state, s_end) and torch.equal(gradient, grads[5]) and all(torch.equal(a, b) for a, b in zip(grads, o))


def test_captured_and_replayed_and_two_at_once():
    from paper_2607_19378_b200 import hyenand as hn
    import os
    if os.environ.get("HYENAND_LIB") == "debug":
        pytest.skip("that build synchronises in every call")
    shape = B, H, Hk, Dk, Dv, L = 1, 2, 2, 64, 64, 1100      # in segments
    a, b = ({k: None if v is None else v.cuda() for k, v in inputs(*shape, torch.bfloat16, "log", s).items()} for s in (12, 13))
    op = hn.DeltaRule(L, B, H, Dk, Dv, Hk, "log", torch.bfloat16)

    def calls(t):
        x = (t["q"], t["k"], t["v"], t["g"], t["beta"])
        y, s_end, marks = op.forward(*x, s0=t["s0"], marks=True)
        return (y, s_end) + op.backward(*x, marks, t["dy"], ds_end=t["ds"])

    want = [[x.clone() for x in calls(t)] for t in (a, b)]
    hold = {k: None if v is None else v.clone() for k, v in a.items()}
    graphs, outs = [torch.cuda.CUDAGraph() for _ in range(2)], []
    for g in graphs:                                          # two graphs of the same shape, in one pool
        with torch.cuda.graph(g, pool=graphs[0].pool() if outs else None):
            outs.append(calls(hold))
    for t, w in ((b, want[1]), (a, want[0])):
        for k, v in hold.items():
            if v is not None:
                v.copy_(t[k])
        for g, o in zip(graphs, outs):
            g.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(p, q) for p, q in zip(o, w))
    got, streams = [None, None], [torch.cuda.Stream() for _ in range(2)]

    def work(i):
        with torch.cuda.stream(streams[i]):
            got[i] = calls((a, b)[i])

    threads = [threading.Thread(target=work, args=(i,)) for i in range(2)]
    for th in threads:
        th.start()
    for th in threads:
        th.join()
    torch.cuda.synchronize()
    assert all(torch.equal(p, q) for g, w in zip(got, want) for p, q in zip(g, w))
    assert hn.hyenand_delta_device_status() == 0


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("decay,Dk,Dv", [("log", 128, 128), ("sigmoid", 50, 97), ("none", 17, 33), ("log", 64, 1)])
def test_tokens_one_by_one(decay, Dk, Dv, dtype):
    """Each token against the oracle's; an entry that has ended keeps its states."""
    from paper_2607_19378_b200 import hyenand as hn
    B, H, Hk, L = 3, 4, 2, 20
    t = inputs(B, H, Hk, Dk, Dv, L, DTYPES[dtype], decay, 14)
    t["lengths"] = torch.tensor([20, 0, 7], dtype=torch.int32)
    op = hn.DeltaRule(1, B, H, Dk, Dv, Hk, decay, DTYPES[dtype])
    state, ys = t["s0"].cuda(), []
    for i in range(L):
        x = [None if t[n] is None else t[n][:, :, i].contiguous().cuda() for n in ("q", "k", "v", "g", "beta")]
        active = (t["lengths"] > i).int().cuda()
        if i % 2:
            ys.append(op.step(*x, state, active=active))
        else:
            new = torch.empty_like(state)
            ys.append(op.step(*x, state, new_state=new, active=active))
            state = new
    ref = od.delta(t["q"], t["k"], t["v"], t["g"], t["beta"], decay, H, Hk, t["s0"], t["lengths"])
    got = {"y": torch.stack([y.cpu() for y in ys], dim=2), "s_end": state.cpu()}
    # fp32 throughout: 2 Dk + 4 roundings a token of what the state holds, twenty tokens
    for name in ("y", "s_end"):
        half = 2.0 ** -8 if got[name].dtype == torch.bfloat16 else 0.0
        assert oracle.rel_l2(got[name], ref[name]) <= half + 20 * (2 * Dk + 4) * 2.0 ** -24, name
    assert torch.equal(got["s_end"][1], t["s0"][1]) and float(got["y"][1].float().abs().max()) == 0.0


def test_thousands_of_tokens_one_by_one_keep_a_decay_next_to_one():
    from paper_2607_19378_b200 import hyenand as hn
    B, H, D, n = 1, 1, 16, 5000
    op = hn.DeltaRule(1, B, H, D)
    g, state = torch.full((B, H), -1e-6, device="cuda"), torch.ones(B, H, D, D, device="cuda")
    zero, beta = torch.zeros(B, D, device="cuda"), torch.zeros(B, H, device="cuda")
    for _ in range(n):
        op.step(zero, zero, zero, g, beta, state)
    # each token rounds the state once (2^-24 of it), with either sign: 5000 of them one way would be 3e-4, as much as sqrt says 4.2e-6
    assert abs(float(state.mean()) / np.exp(-1e-6 * n) - 1) < 1e-4


def test_elements_past_two_to_the_31():
    """The last head of tensors of 2^31 elements and more: the same numbers as that head alone."""
    from paper_2607_19378_b200 import hyenand as hn
    import os
    if os.environ.get("HYENAND_LIB") == "debug":
        pytest.skip("minutes with range checks, and no kernel that smaller ones leave out")
    H, D, L = 17, 128, 1 << 20
    gen = torch.Generator(device="cuda").manual_seed(15)
    n = lambda *s: torch.randn(s, generator=gen, device="cuda", dtype=torch.bfloat16)
    q, k, v = (n(1, H * D, L) for _ in range(3))
    for x in (q, k):
        for h in range(H):
            part = x[:, h * D:(h + 1) * D]
            part /= part.float().norm(dim=1, keepdim=True).to(x.dtype)
    g, beta = -torch.rand((1, H, L), generator=gen, device="cuda") * 0.1, torch.rand((1, H, L), generator=gen, device="cuda")
    y, s_end = hn.DeltaRule(L, 1, H, D, dtype=torch.bfloat16).forward(q, k, v, g, beta)
    cut = lambda x, d: x[:, -d:].contiguous()
    y1, s1 = hn.DeltaRule(L, 1, 1, D, dtype=torch.bfloat16).forward(cut(q, D), cut(k, D), cut(v, D), cut(g, 1), cut(beta, 1))
    last = y[:, -D:]
    err = sum(float((a.float() - b.float()).square().sum()) for a, b in zip(last.chunk(16, 2), y1.chunk(16, 2)))
    size = sum(float(b.float().square().sum()) for b in y1.chunk(16, 2))
    assert (err / size) ** 0.5 <= 2 * 2.0 ** -8 and float((s_end[:, -1] - s1[:, 0]).norm() / s1.norm()) <= 2 * 7 * 2.0 ** -16
