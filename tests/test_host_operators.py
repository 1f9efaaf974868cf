"""Refusals of the recurrence's, the residual block's and dropout's entry points, without a GPU: addresses are compared and checked
on the host before anything is launched, so plain numbers stand for buffers."""
import ctypes

import pytest
import torch

A = [(i + 1) << 24 for i in range(24)]           # distinct 16-byte-aligned addresses, 16 MiB apart


@pytest.fixture(scope="module")
def hn():
    from paper_2607_19378_b200.build import build
    build()
    from paper_2607_19378_b200 import hyenand
    return hyenand


def refused(hn, code, word):
    assert code in (hn.HYENAND_ERR_INVALID_ARG, hn.HYENAND_ERR_UNSUPPORTED) and word in hn.hyenand_last_error(), (code, hn.hyenand_last_error())


def forward_args(**kw):
    a = dict(B=2, C=3, L=40, decay=1, dtype=0, q=A[0], k=A[1], v=A[2], g=A[3], s0=None, lengths=None, y=A[4], s_end=None, marks=None, workspace=None, stream=None)
    a.update(kw)
    return list(a.values())


@pytest.mark.parametrize("change,word", [
    (dict(B=0), "B, C and L"), (dict(C=0), "B, C and L"), (dict(L=0), "B, C and L"), (dict(L=-5), "B, C and L"), (dict(L=(1 << 30) + 1), "2^30"),
    (dict(B=1 << 15, C=(1 << 13) + 1, L=1), "2^28"), (dict(decay=3), "decay"), (dict(decay=-1), "decay"), (dict(dtype=2), "dtype"),
    (dict(q=None), "non-NULL"), (dict(g=None), "non-NULL"), (dict(y=None), "non-NULL"), (dict(v=A[2] + 8), "aligned"), (dict(s0=A[5] + 2), "aligned"),
    (dict(y=A[0]), "overlaps"), (dict(y=A[3] + 944), "overlaps"), (dict(s_end=A[4] + 16), "overlaps"), (dict(s0=A[5], s_end=A[5] + 4), "overlaps"),
    (dict(marks=A[2] - 16), "overlaps"), (dict(lengths=A[6], s_end=A[6]), "overlaps"),
    (dict(L=100000), "workspace"), (dict(L=100000, workspace=A[7] + 8), "aligned"), (dict(L=100000, workspace=A[3]), "overlaps")], ids=str)
def test_recurrence_forward_refuses(hn, change, word):
    refused(hn, hn.lib().hyenand_recurrence_forward(*forward_args(**change)), word)


@pytest.mark.parametrize("change,word", [
    (dict(marks=None), "non-NULL"), (dict(dy=None), "non-NULL"), (dict(dq=None), "non-NULL"), (dict(dg=A[3]), "overlaps"), (dict(dk=A[7]), "overlaps"),
    (dict(ds0=A[5]), "overlaps"), (dict(dy=A[6] + 4), "aligned"), (dict(L=0), "B, C and L")], ids=str)
def test_recurrence_backward_refuses(hn, change, word):
    a = dict(B=2, C=3, L=40, decay=2, dtype=1, q=A[0], k=A[1], v=A[2], g=A[3], lengths=None, marks=A[5], dy=A[6], ds_end=None, dq=A[7], dk=A[8],
             dv=A[9], dg=A[10], ds0=None, workspace=None, stream=None)
    a.update(change)
    refused(hn, hn.lib().hyenand_recurrence_backward(*a.values()), word)


@pytest.mark.parametrize("change,word", [(dict(state=None), "non-NULL"), (dict(new_state=None), "non-NULL"), (dict(y=A[4]), "overlaps"),
                                         (dict(new_state=A[4] + 16), "overlaps"), (dict(B=0), "B, C and L"), (dict(decay=9), "decay")], ids=str)
def test_recurrence_step_refuses(hn, change, word):
    a = dict(B=4, C=30, decay=0, dtype=0, q=A[0], k=A[1], v=A[2], g=A[3], state=A[4], active=None, y=A[5], new_state=A[4], stream=None)
    a.update(change)
    refused(hn, hn.lib().hyenand_recurrence_step(*a.values()), word)


BLOCK = dict(B=2, C=3, T=40, dtype=0, x=A[0], m=A[1], z=A[2], g_post=A[3], scale=A[4], g_pre=A[5], eps=1e-6, gate=2, p=0.1, rng=A[6], site=0)


@pytest.mark.parametrize("change,word", [
    (dict(B=0), "B, C and T"), (dict(T=0), "B, C and T"), (dict(T=(1 << 30) + 1), "2^30"), (dict(C=(1 << 20) + 1), "2^20"),
    (dict(B=1 << 12, C=1 << 10, T=(1 << 18) + 1), "2^40"), (dict(dtype=5), "dtype"), (dict(gate=3), "gate"), (dict(gate=0), "z is given"), (dict(z=None), "z is given"),
    (dict(x=None), "x and m"), (dict(eps=0.0), "eps"), (dict(eps=-1.0), "eps"), (dict(eps=float("nan")), "eps"), (dict(eps=float("inf")), "eps"),
    (dict(p=1.0), "p must"), (dict(p=-0.1), "p must"), (dict(p=float("nan")), "p must"), (dict(rng=None), "rng"), (dict(r=None), "r must"),
    (dict(n=None), "n is given"), (dict(g_pre=None), "n is given"), (dict(r=A[0]), "overlaps"), (dict(n=A[7]), "overlaps"), (dict(stats=A[2]), "overlaps"),
    (dict(m=A[1] + 4), "aligned"), (dict(rng=A[6] + 8), "aligned")], ids=str)
def test_block_forward_refuses(hn, change, word):
    a = dict(BLOCK, r=A[7], n=A[8], stats=None, stream=None)
    a.update(change)
    refused(hn, hn.lib().hyenand_block_forward(*a.values()), word)


@pytest.mark.parametrize("change,word", [
    (dict(dx=None), "dx, dm"), (dict(workspace=None), "dx, dm"), (dict(dz=None), "dz is given"), (dict(z=None, gate=0), "dz is given"), (dict(dn=None), "dn is given"),
    (dict(g_pre=None), "dn is given"), (dict(stats=None), "stats"), (dict(g_post=None), "weight"), (dict(scale=None), "weight"),
    (dict(dr=None, dn=None, g_pre=None, dg_pre=None), "dr or dn"), (dict(dm=A[1]), "overlaps"), (dict(workspace=A[0]), "overlaps"), (dict(dg_pre=A[14]), "overlaps")],
    ids=str)
def test_block_backward_refuses(hn, change, word):
    a = dict(BLOCK, stats=A[7], dr=A[8], dn=A[9], dx=A[10], dm=A[11], dz=A[12], dg_post=A[13], dscale=A[14], dg_pre=A[15], workspace=A[16], stream=None)
    a.update(change)
    refused(hn, hn.lib().hyenand_block_backward(*a.values()), word)


@pytest.mark.parametrize("change,word", [(dict(n=0), "n must"), (dict(n=-3), "n must"), (dict(dtype=2), "dtype"), (dict(x=None), "non-NULL"), (dict(rng=None), "non-NULL"),
                                         (dict(p=1.0), "p must"), (dict(p=-1e-3), "p must"), (dict(y=A[0] + 16), "overlaps"), (dict(y=A[2]), "overlaps"),
                                         (dict(x=A[0] + 4), "aligned")], ids=str)
def test_dropout_refuses(hn, change, word):
    a = dict(n=1000, dtype=0, x=A[0], p=0.5, rng=A[2], site=0, y=A[1], stream=None)
    a.update(change)
    refused(hn, hn.lib().hyenand_dropout(*a.values()), word)


def test_sizes(hn):
    assert [hn.hyenand_recurrence_marks(L) for L in (0, 1, 249, 250, 505, 506, 1 << 30, (1 << 30) + 1)] == [0, 1, 1, 2, 2, 3, (1 << 22) + 1, 0]
    assert [hn.hyenand_recurrence_workspace_bytes(*a) for a in ((1, 24, 0, 0), (1, 0, 9, 0), (1, 24, 1000, 0), (64, 64, 1 << 20, 1))] == [0] * 4
    assert 16 * 24 * 2 <= hn.hyenand_recurrence_workspace_bytes(1, 24, 100003, 0) <= 1 << 16
    assert hn.hyenand_block_workspace_bytes(1, 8, 4, 0) >= 3 * 8 * 4 and hn.hyenand_block_workspace_bytes(1, 0, 4, 0) == 0


def test_classes_refuse_tensors(hn):
    """Tensors that are not the handle's: ValueError before the library is called."""
    rec = hn.Recurrence(8, 2, 3)
    t = torch.zeros(2, 3, 8)
    with pytest.raises(ValueError, match="q must be"):
        rec.forward(t, t, t, t)                              # on the host
    with pytest.raises(ValueError, match="q must be"):
        rec.step(t, t, t, t, t)
    with pytest.raises(ValueError, match="x must be"):
        hn.Block((8,), 2, 3).forward(t, t)
    with pytest.raises(ValueError, match="x must be"):
        hn.Dropout(0.5)(t, torch.zeros(2, dtype=torch.int64))
    with pytest.raises(ValueError, match="float32 or bfloat16"):
        hn.Dropout(0.5)(t.double(), torch.zeros(2, dtype=torch.int64))
    with pytest.raises(TypeError, match="q must be a tensor"):
        rec.forward(None, t, t, t)
    for bad in (dict(L=0), dict(B=0), dict(C=0), dict(L=(1 << 30) + 1)):
        with pytest.raises(ValueError):
            hn.Recurrence(**dict(dict(L=8, B=2, C=3), **bad))
    with pytest.raises(KeyError):
        hn.Recurrence(8, 2, 3, decay="linear")
    with pytest.raises(ValueError):
        hn.Block((8, 0), 2, 3)
