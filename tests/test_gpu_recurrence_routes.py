"""Every way in which the recurrence walks many or long rows, on ragged batches with a state before and a gradient behind, against
oracle/recurrence.py.  Bounds: those of test_gpu_recurrence.py."""
import pytest
import torch

from oracle import recurrence as orec
from test_gpu_recurrence import DTYPES, compare, inputs, run

pytestmark = pytest.mark.gpu


# rows of a few tiles by a warp each, the number of rows no multiple of the four of a CTA; two warps a row in several waves; 192 lanes
# forward, 128 forward and 256 backward, 256 forward
@pytest.mark.parametrize("decay", ["value", "log", "sigmoid"])
@pytest.mark.parametrize("B,C,L,dtype,lengths", [
    (3, 601, 1531, "bf16", [1531, 0, 700]), (3, 601, 1536, "bf16", [1, 1536, 513]), (3, 601, 777, "f32", [0, 777, 256]), (3, 601, 1024, "f32", [1024, 255, 1]),
    (3, 601, 2500, "bf16", [2500, 0, 1025]), (2, 250, 5003, "bf16", [5003, 4000]), (2, 350, 4500, "bf16", [100, 4500]), (3, 100, 4100, "f32", [4100, 0, 4099])],
    ids=str)
def test_ragged_batches(B, C, L, dtype, lengths, decay):
    t = inputs(B, C, L, DTYPES[dtype], decay, B * L)
    t["lengths"] = torch.tensor(lengths, dtype=torch.int32)
    ref = orec.recurrence(t["q"], t["k"], t["v"], t["g"], decay, t["s0"], t["lengths"], t["dy"], t["ds"])
    for n in ("q", "k", "v", "g", "dy"):
        for b, m in enumerate(lengths):
            t[n][b, :, m:] = float("nan")
    got = run(t, L, B, C, DTYPES[dtype], decay)
    compare(got, ref, L)
    for b, m in enumerate(lengths):
        if m == 0:
            assert torch.equal(got["s_end"][b], t["s0"][b]) and torch.equal(got["ds0"][b], t["ds"][b])


# prompts of a batch, the long-context layers: a few rows of each, first, last and between, and the same bits twice
@pytest.mark.parametrize("B,C,L,dtype,decay,ragged", [(16, 768, 2000, "bf16", "sigmoid", True), (2, 256, 65536, "bf16", "log", False),
                                                      (2, 256, 262144, "bf16", "log", False), (8, 768, 8192, "bf16", "sigmoid", True)], ids=str)
def test_full_sizes(B, C, L, dtype, decay, ragged):
    from paper_2607_19378_b200 import hyenand as hn
    gen, dt = torch.Generator(device="cuda").manual_seed(L), DTYPES[dtype]
    n = lambda *s: torch.randn(s, generator=gen, device="cuda")
    t = {k: n(B, C, L).to(dt) for k in ("q", "k", "v", "dy")}
    rate = torch.exp(-6.9 * torch.rand((1, C, 1), generator=gen, device="cuda"))
    t["g"] = (n(B, C, L) + 6 * rate if decay == "sigmoid" else -rate * n(B, C, L).abs()).to(dt)
    s0, ds = n(B, C), n(B, C)
    lengths = torch.randint(L // 3, L + 1, (B,), generator=gen, device="cuda", dtype=torch.int32) if ragged else None
    op = hn.Recurrence(L, B, C, decay, dt)

    def once():
        y, end, marks = op.forward(t["q"], t["k"], t["v"], t["g"], s0=s0, lengths=lengths, marks=True)
        return (y, end) + op.backward(t["q"], t["k"], t["v"], t["g"], marks, t["dy"], ds_end=ds, lengths=lengths)
    out = once()
    assert all(torch.equal(a, b) for a, b in zip(out, once()))
    rows = torch.tensor([0, 1, C // 2 + 1, C - 1])
    for b in (0, B - 1):
        part = {k: v[b:b + 1, rows].cpu() for k, v in t.items()}
        ref = orec.recurrence(part["q"], part["k"], part["v"], part["g"], decay, s0[b:b + 1, rows].cpu(), None if lengths is None else lengths[b:b + 1].cpu(),
                              part["dy"], ds[b:b + 1, rows].cpu())
        compare({k: v[b:b + 1, rows].cpu() for k, v in zip(("y", "s_end", "dq", "dk", "dv", "dg", "ds0"), out)}, ref, L)
    assert hn.hyenand_recurrence_device_status() == 0
