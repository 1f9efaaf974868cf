"""Heads, the delta rule and the residual block together, as a layer uses them: queries and keys normalised and turned by their place on a grid,
the rule over the grid's tokens in order, its result gated into the stream; forward and gradients of the chain against torch autograd in
64 bits, and the tokens again one by one.

Tolerance: fp32 throughout; each operator is within 1e-5 of its exact value in the 2-norm and three of them follow one another in either
direction: 4e-5."""
import pytest
import torch

import oracle

pytestmark = pytest.mark.gpu


def test_training_step_and_generation():
    from paper_2607_19378_b200 import hyenand as hn
    B, H, Hk, D, Dv, dims, axes = 2, 4, 2, 24, 20, (9, 13), (5, 6)
    L, C = dims[0] * dims[1], H * Dv
    gen = torch.Generator().manual_seed(41)
    n = lambda *s: torch.randn(s, generator=gen)
    t = dict(q=n(B, Hk * D, *dims), k=n(B, Hk * D, *dims), v=n(B, C, L), g=1 + n(B, H, L), beta=torch.sigmoid(n(B, H, L)), x=n(B, C, L), z=n(B, C, L), gq=1 + 0.1 * n(D),
             gk=1 + 0.1 * n(D), gp=1 + 0.1 * n(C), sc=0.5 + 0.1 * n(C), gn=1 + 0.1 * n(C))
    do, dn = n(B, C, L), n(B, C, L)
    d = {k: a.cuda() for k, a in t.items()}
    heads, rule, blk = hn.Heads(dims, B, Hk, Hk, D, norm="l2", axes=axes), hn.DeltaRule(L, B, H, D, Dv, Hk, "sigmoid"), hn.Block((L,), B, C, gate="silu")
    flat, w = lambda a: a.view(B, -1, L), dict(z=d["z"], g_post=d["gp"], scale=d["sc"], g_pre=d["gn"])
    q, k = heads.forward(d["q"], d["k"], d["gq"], d["gk"])
    x = (flat(q), flat(k), d["v"], d["g"], d["beta"])
    m, s_end, marks = rule.forward(*x, marks=True)
    r, nn, st = blk.forward(d["x"], m, stats=True, **w)
    dx, dm, dz, dgp, dsc, dgn = blk.backward(d["x"], m, st, dr=do.cuda(), dn=dn.cuda(), **w)
    dq, dk, dv, dg, dbeta, _ = rule.backward(*x, marks, dm)
    dq, dk, dgq, dgk = heads.backward(d["q"], d["k"], dq.view(q.shape), dk.view(k.shape), d["gq"], d["gk"])
    got = dict(q=dq, k=dk, v=dv, g=dg, beta=dbeta, x=dx, z=dz, gq=dgq, gk=dgk, gp=dgp, sc=dsc, gn=dgn)

    leaf = {k: a.double().requires_grad_(True) for k, a in t.items()}
    from oracle import heads as oh
    ang = torch.tensor(oh.turns(dims, axes, D, 10000.0))[:, None]

    def turned(a, w):
        a = a.reshape(B, Hk, D, L)
        a = a / torch.sqrt((a ** 2).sum(2, keepdim=True) + 1e-6) * w.view(1, 1, D, 1)
        lo, hi = a[:, :, :D // 2], a[:, :, D // 2:]
        return torch.cat([lo * torch.cos(ang) - hi * torch.sin(ang), lo * torch.sin(ang) + hi * torch.cos(ang)], dim=2).repeat_interleave(H // Hk, dim=1)

    Q, K, V = turned(leaf["q"], leaf["gq"]), turned(leaf["k"], leaf["gk"]), leaf["v"].reshape(B, H, Dv, L)
    S, rows = torch.zeros(B, H, Dv, D, dtype=torch.float64), []
    for i in range(L):
        S = torch.sigmoid(leaf["g"])[:, :, i, None, None] * S
        u = leaf["beta"][:, :, i, None] * (V[..., i] - torch.einsum("bhij,bhj->bhi", S, K[..., i]))
        S = S + u[..., :, None] * K[..., i][..., None, :]
        rows.append(torch.einsum("bhij,bhj->bhi", S, Q[..., i]).reshape(B, C))
    mm = torch.stack(rows, dim=-1)
    rms = lambda a, g: a / torch.sqrt((a ** 2).mean(1, keepdim=True) + 1e-6) * g.view(1, -1, 1)
    rr = leaf["x"] + leaf["sc"].view(1, C, 1) * torch.nn.functional.silu(leaf["z"]) * rms(mm, leaf["gp"])
    out = rms(rr, leaf["gn"])
    want = dict(zip(leaf, torch.autograd.grad((rr * do).sum() + (out * dn).sum(), list(leaf.values()))))
    assert oracle.rel_l2(r.cpu(), rr.detach().numpy()) < 4e-5 and oracle.rel_l2(nn.cpu(), out.detach().numpy()) < 4e-5
    for name, a in got.items():
        assert oracle.rel_l2(a.cpu(), want[name].numpy()) < 4e-5, name

    # generation: the same tokens one by one, each at its own place
    one_heads, one = hn.Heads((1, 1), B, Hk, Hk, D, norm="l2", axes=axes), hn.DeltaRule(1, B, H, D, Dv, Hk, "sigmoid")
    state, ys = torch.zeros_like(s_end), []
    for i in range(L):
        at = torch.tensor([i // dims[1], i % dims[1]], dtype=torch.int32, device="cuda").view(1, 2, 1, 1).expand(B, 2, 1, 1).contiguous()
        cut = lambda a: a.reshape(B, -1, L)[:, :, i].contiguous()
        q1, k1 = one_heads.forward(cut(d["q"]).view(B, -1, 1, 1), cut(d["k"]).view(B, -1, 1, 1), d["gq"], d["gk"], positions=at)
        ys.append(one.step(q1.view(B, -1), k1.view(B, -1), cut(d["v"]), cut(d["g"]), cut(d["beta"]), state))
    assert oracle.rel_l2(torch.stack(ys, dim=2).cpu(), mm.detach().numpy()) < 4e-5 and oracle.rel_l2(state.cpu(), S.detach().numpy()) < 4e-5
