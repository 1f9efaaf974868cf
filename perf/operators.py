"""Operators of a residual block around the long convolution, as they are measured.

Three operators on the library's layout [B, C, L_1..L_N], with what each of them computes written out in `run`'s plain
forms (`own` false) and called through the library's entry points where `own` is true:

    recurrence   the gated linear recurrence  s_t = a_t s_{t-1} + k_t v_t,  y_t = q_t s_t,  whose decay a_t comes from a gate
                 per token; kinds: "step" (one token against a kept state), "scan" (a sequence, from a state to a state),
                 "scan_train" (a sequence and its gradients)
    block        what stands between two mixers of a residual stream x: the mixer's output m normalised, gated by z, dropped
                 out and scaled into the stream, the new stream normalised for the next mixer; kinds: "block", "block_train"
    dropout      y = x keep / (1 - p), the mask drawn from counters; kind: "dropout" (its backward is the same call)

A case is a dict of plain values.  `exact` evaluates the definitions in 64 bits, by loops of its own.
"""
import math

import numpy as np
import torch

own = False

_EPS = 1e-6
_GATES = ("none", "sigmoid", "silu")
_DECAYS = ("value", "log", "sigmoid")


def _scan_case(name, kind, L, B, C, dtype, decay, ragged):
    c = {"op": "recurrence", "kind": kind, "dims": str(L), "B": B, "C": C, "dtype": dtype, "decay": decay, "ragged": ragged}
    return dict(c, name=name) if name else c


def _block_case(name, kind, dims, B, C, dtype, gate, post, p):
    c = {"op": "block", "kind": kind, "dims": dims, "B": B, "C": C, "dtype": dtype, "gate": gate, "post": post, "p": p}
    return dict(c, name=name) if name else c


def _dropout_case(name, dims, B, C, dtype, p):
    c = {"op": "dropout", "kind": "dropout", "dims": dims, "B": B, "C": C, "dtype": dtype, "p": p}
    return dict(c, name=name) if name else c


def listed():
    return [
        # one generated token for a batch of 32 sequences, some of which have ended
        _scan_case("step", "step", 1, 32, 768, "bf16", "log", True),
        # prompts of unequal length, carried on from a state: an ordinary context, as the causal convolution's
        _scan_case("scan_prompts", "scan", 2000, 16, 768, "bf16", "sigmoid", True),
        # long-context genomics layer, the benchmark's sequence
        _scan_case("scan_genomics", "scan", 262144, 2, 256, "bf16", "log", False),
        # few rows of an odd length, fp32: one sequence of a narrow layer
        _scan_case("scan_narrow", "scan", 100003, 1, 24, "f32", "sigmoid", False),
        # training step of a long-context layer
        _scan_case("train_long", "scan_train", 65536, 2, 256, "bf16", "log", False),
        # training step on a padded batch of short sequences with an odd row length, fp32, decays given as they are
        _scan_case("train_padded", "scan_train", 1531, 5, 97, "f32", "value", True),
        # between two mixers at inference, ViT-like grid of 14x14 patches and a row of register tokens
        _block_case("block_tokens", "block", "15x14", 32, 768, "bf16", "silu", True, 0.0),
        # training step on the benchmark's vision grid, with dropout
        _block_case("block_vision", "block_train", "64x64", 16, 768, "bf16", "silu", True, 0.1),
        # training step on an odd grid, gate without a norm of its own
        _block_case("block_odd", "block_train", "31x33", 8, 200, "bf16", "sigmoid", False, 0.0),
        # training step on volumes, few channels and many tokens, fp32
        _block_case("block_volume", "block_train", "96x96x96", 1, 64, "f32", "none", True, 0.0),
        # dropout of a small fp32 grid, where the launch is what it takes
        _dropout_case("dropout_small", "32x32", 1, 8, "f32", 0.2),
        # dropout of the vision grid's activations
        _dropout_case("dropout_vision", "64x64", 16, 768, "bf16", 0.1),
    ]


def _log(rng, lo, hi):
    return math.exp(rng.uniform(math.log(lo), math.log(hi)))


def draw(rng):
    """Sequences of 1 to 262144 positions, planes of 4 to 256 and volumes of 4 to 96 per axis, 1 to 2048 channels, odd extents
    among them; the batch follows from a budget of elements."""
    kind = rng.choice(["step", "scan", "scan", "scan_train", "scan_train", "block", "block_train", "block_train", "dropout"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    budget = _log(rng, 1 << 14, {"scan": 1 << 25, "scan_train": 1 << 23, "block_train": 1 << 24}.get(kind, 1 << 24))
    if kind == "step":
        return _scan_case("", kind, 1, round(_log(rng, 1, 256)), round(_log(rng, 8, 4096)), dtype, rng.choice(_DECAYS), rng.random() < 0.5)
    if kind in ("scan", "scan_train"):
        L = max(1, round(_log(rng, 1, min(262144, budget / 8))))
        rows = max(1, int(budget / L))
        B = max(1, min(rows, round(_log(rng, 1, 32))))
        C = max(1, min(2048, rows // B))
        return _scan_case("", kind, L, B, C, dtype, rng.choice(_DECAYS), rng.random() < 0.5)
    ndim = rng.choice([1, 2, 2, 3])
    top, low = {1: 16384, 2: 256, 3: 96}[ndim], {1: 1, 2: 4, 3: 4}[ndim]
    base = _log(rng, low, min(top, max(low, (budget / 16) ** (1.0 / ndim))))
    dims = [max(low, min(top, round(base * _log(rng, 0.7, 1.4)))) for _ in range(ndim)]
    slices = max(1, int(budget / math.prod(dims)))
    C = max(1, min(slices, 2048, round(_log(rng, 8, 2048))))
    B = max(1, min(64, slices // C))
    text = "x".join(str(d) for d in dims)
    if kind == "dropout":
        return _dropout_case("", text, B, C, dtype, rng.choice([0.05, 0.1, 0.2, 0.5]))
    return _block_case("", kind, text, B, C, dtype, rng.choice(_GATES), rng.random() < 0.7,
                       rng.choice([0.0, 0.1, 0.2]) if kind == "block_train" else 0.0)


def _dims(case):
    return tuple(int(d) for d in case["dims"].split("x"))


def _torch_dtype(case):
    return torch.float32 if case["dtype"] == "f32" else torch.bfloat16


def prepare(case, seed):
    dev = "cuda"
    gen = torch.Generator(device=dev)
    gen.manual_seed(seed * 1000003 + 29)
    dt, dims, B, C = _torch_dtype(case), _dims(case), case["B"], case["C"]
    shape = (B, C) + dims

    def normal(sh=shape, dtype=dt):
        return torch.randn(sh, generator=gen, device=dev).to(dtype)

    def uniform(sh, lo, hi):
        return torch.rand(sh, generator=gen, device=dev) * (hi - lo) + lo

    s = {"case": case}
    if case["op"] == "recurrence":
        L = dims[0]
        if case["kind"] == "step":
            shape = (B, C)
        s["q"], s["k"], s["v"] = normal(shape), normal(shape), normal(shape)
        # a memory of its own for every channel, from a few tokens to thousands, modulated by every token
        chan = (1, C) + (1,) * (len(shape) - 2)
        if case["decay"] == "log":
            rate = torch.exp(uniform(chan, math.log(1e-3), math.log(1.0)))
            g = -rate * torch.log1p(torch.exp(normal(shape, torch.float32)))
        else:
            g = uniform(chan, 0.0, 6.0) + normal(shape, torch.float32)
            if case["decay"] == "value":
                g = 1.0 / (1.0 + torch.exp(-g))
        s["g"] = g.to(dt)
        s["s0"] = normal((B, C), torch.float32)
        s["lengths"] = None
        if case["ragged"]:
            n = torch.floor(uniform((B,), 0.4, 1.0) * (L + 1)) if L > 1 else (uniform((B,), 0.0, 1.0) < 0.9).float()
            s["lengths"] = n.clamp(0, L).to(torch.int32)
        if case["kind"] == "scan_train":
            s["dy"] = normal()
            s["ds"] = normal((B, C), torch.float32)
        return s
    s["rng"] = torch.tensor([0x5DEECE66D + 7919 * seed, 1 + seed], dtype=torch.int64, device=dev)       # seed and step of the generator
    s["x"] = normal()
    if case["op"] == "dropout":
        return s
    s["m"] = normal() * 2
    s["z"] = normal() if case["gate"] != "none" else None
    s["g_post"] = 1.0 + 0.1 * normal((C,), torch.float32) if case["post"] else None
    s["scale"] = uniform((C,), 0.1, 1.0)
    s["g_pre"] = 1.0 + 0.1 * normal((C,), torch.float32)
    if case["kind"] == "block_train":
        s["dr"], s["dn"] = normal(), normal()
    return s


# ---- the framework's calls -----------------------------------------------------------------------------------------

def _op(s):
    """The object a program keeps: made once, on the first pass."""
    if "own_op" not in s:
        from paper_2607_19378_b200 import hyenand as hn
        c = s["case"]
        if c["op"] == "recurrence":
            s["own_op"] = hn.Recurrence(_dims(c)[0], c["B"], c["C"], decay=c["decay"], dtype=_torch_dtype(c))
        elif c["op"] == "block":
            s["own_op"] = hn.Block(_dims(c), c["B"], c["C"], dtype=_torch_dtype(c), gate=c["gate"], eps=_EPS, p=c["p"])
        else:
            s["own_op"] = hn.Dropout(c["p"])
        if c["kind"] == "step":
            s["state"] = torch.empty_like(s["s0"])            # the states before and after a token, kept side by side
    return s["own_op"]


def _run_own(s):
    c, op = s["case"], _op(s)
    if c["kind"] == "step":
        return {"y": op.step(s["q"], s["k"], s["v"], s["g"], s["s0"], new_state=s["state"], active=s["lengths"]), "s_end": s["state"]}
    if c["kind"] == "scan":
        y, s_end = op.forward(s["q"], s["k"], s["v"], s["g"], s0=s["s0"], lengths=s["lengths"])
        return {"y": y, "s_end": s_end}
    if c["kind"] == "scan_train":
        y, s_end, marks = op.forward(s["q"], s["k"], s["v"], s["g"], s0=s["s0"], lengths=s["lengths"], marks=True)
        dq, dk, dv, dg, ds0 = op.backward(s["q"], s["k"], s["v"], s["g"], marks, s["dy"], ds_end=s["ds"], lengths=s["lengths"])
        return {"y": y, "s_end": s_end, "dq": dq, "dk": dk, "dv": dv, "dg": dg, "ds0": ds0}
    if c["kind"] == "dropout":
        return op(s["x"], s["rng"])
    weights = {"z": s["z"], "g_post": s["g_post"], "scale": s["scale"], "g_pre": s["g_pre"], "rng": s["rng"] if c["p"] else None}
    if c["kind"] == "block":
        r, n = op.forward(s["x"], s["m"], **weights)
        return {"r": r, "n": n}
    r, n, stats = op.forward(s["x"], s["m"], stats=True, **weights)
    dx, dm, dz, dg_post, dscale, dg_pre = op.backward(s["x"], s["m"], stats, dr=s["dr"], dn=s["dn"], **weights)
    return _block_outputs(r, n, dx, dm, dz, dg_post, dscale, dg_pre)


def _block_outputs(r, n, dx, dm, dz, dg_post, dscale, dg_pre):
    out = {"r": r, "n": n, "dx": dx, "dm": dm, "dscale": dscale, "dg_pre": dg_pre}
    if dz is not None:
        out["dz"] = dz
    if dg_post is not None:
        out["dg_post"] = dg_post
    return out


# ---- plain forms ---------------------------------------------------------------------------------------------------

def _linear_scan(a, u, s0):
    """s_t = a_t s_{t-1} + u_t along the last axis from s0: spans doubled until they reach the whole row."""
    S = u.clone()
    S[..., 0] += a[..., 0] * s0
    A = a.clone()
    d, L = 1, a.shape[-1]
    while d < L:
        S[..., d:] += A[..., d:] * S[..., :-d].clone()
        if 2 * d < L:
            A[..., d:] *= A[..., :-d].clone()
        d *= 2
    return S


def _decay(g, kind):
    return g if kind == "value" else torch.exp(g) if kind == "log" else 1.0 / (1.0 + torch.exp(-g))


def _plain_recurrence(s):
    c = s["case"]
    dt = _torch_dtype(c)
    step = c["kind"] == "step"
    q, k, v, g = ((t.unsqueeze(-1) if step else t).float() for t in (s["q"], s["k"], s["v"], s["g"]))
    L = q.shape[-1]
    live = None
    if s["lengths"] is not None:
        live = torch.arange(L, device=q.device)[None, None, :] < s["lengths"][:, None, None]
    a, u = _decay(g, c["decay"]), k * v
    if live is not None:
        a, u = torch.where(live, a, 1.0), torch.where(live, u, 0.0)
    S = _linear_scan(a, u, s["s0"])
    y = q * S
    if live is not None:
        y = torch.where(live, y, 0.0)
    out = {"y": y.to(dt).squeeze(-1) if step else y.to(dt), "s_end": S[..., -1].clone()}
    if c["kind"] != "scan_train":
        return out
    dy = s["dy"].float()
    w = q * dy
    if live is not None:
        w, dy = torch.where(live, w, 0.0), torch.where(live, dy, 0.0)
    ahead = torch.cat([a[..., 1:], torch.ones_like(a[..., :1])], dim=-1)             # a_{t+1}; the state's gradient comes in behind the row
    lam = _linear_scan(ahead.flip(-1), w.flip(-1), s["ds"]).flip(-1)
    before = torch.cat([s["s0"][..., None], S[..., :-1]], dim=-1)
    da = lam * before
    dg = da if c["decay"] == "value" else da * a if c["decay"] == "log" else da * a / (1.0 + torch.exp(g))
    dk, dv = lam * v, lam * k
    if live is not None:
        dk, dv, dg = (torch.where(live, t, 0.0) for t in (dk, dv, dg))
    return dict(out, dq=(dy * S).to(dt), dk=dk.to(dt), dv=dv.to(dt), dg=dg.to(dt), ds0=a[..., 0] * lam[..., 0])


_M32 = 0xFFFFFFFF


def _threshold(p):
    return min(65535, int(p * 65536 + 0.5))


def _philox(counters, rng, site):
    """Four words of 32 bits for every counter: Philox4x32-10, counter (index, index >> 32, step, site), key = seed."""
    c0, c1 = counters & _M32, counters >> 32
    c2, c3 = (rng[1] & _M32).expand_as(c0), torch.full_like(c0, site)
    k0, k1 = rng[0] & _M32, (rng[0] >> 32) & _M32
    for _ in range(10):
        p0, p1 = c0 * 0xD2511F53, c2 * 0xCD9E8D57
        c0, c1, c2, c3 = ((p1 >> 32) & _M32) ^ c1 ^ k0, p1 & _M32, ((p0 >> 32) & _M32) ^ c3 ^ k1, p0 & _M32
        k0, k1 = (k0 + 0x9E3779B9) & _M32, (k1 + 0xBB67AE85) & _M32
    return c0, c1, c2, c3


def _drop_factor(like, p, rng, site=0):
    """keep / (1 - p) for every element in memory order: 16 bits each, eight elements a counter."""
    n = like.numel()
    words = _philox(torch.arange((n + 7) // 8, device=like.device), rng, site)
    halves = torch.stack([h for w in words for h in (w & 0xFFFF, w >> 16)], dim=-1).reshape(-1)[:n]
    thr = _threshold(p)
    return (halves >= thr).float().mul_(65536.0 / (65536 - thr)).reshape(like.shape)


def _act(z, gate):
    sg = 1.0 / (1.0 + torch.exp(-z))
    return sg if gate == "sigmoid" else z * sg


def _act_grad(z, gate):
    sg = 1.0 / (1.0 + torch.exp(-z))
    return sg / (1.0 + torch.exp(z)) if gate == "sigmoid" else sg * (1.0 + z / (1.0 + torch.exp(z)))


def _plain_block(s):
    c = s["case"]
    dt = _torch_dtype(c)
    flat = (c["B"], c["C"], -1)
    x, m = s["x"].float().reshape(flat), s["m"].float().reshape(flat)
    z = s["z"].float().reshape(flat) if s["z"] is not None else None
    col = lambda t: t[None, :, None]
    rho_m = torch.rsqrt(torch.mean(m * m, dim=1, keepdim=True) + _EPS) if c["post"] else None
    mh = m * rho_m if c["post"] else m
    mn = mh * col(s["g_post"]) if c["post"] else m
    w = mn * _act(z, c["gate"]) if z is not None else mn
    D = _drop_factor(x, c["p"], s["rng"]) if c["p"] else None
    wd = w * D if D is not None else w
    r = x + col(s["scale"]) * wd
    rho_r = torch.rsqrt(torch.mean(r * r, dim=1, keepdim=True) + _EPS)
    rh = r * rho_r
    shape = s["x"].shape
    out = (r.to(dt).reshape(shape), (rh * col(s["g_pre"])).to(dt).reshape(shape))
    if c["kind"] == "block":
        return {"r": out[0], "n": out[1]}
    dr, dn = s["dr"].float().reshape(flat), s["dn"].float().reshape(flat)
    dg_pre = torch.sum((dn * rh).double(), dim=(0, 2)).float()
    e = dn * col(s["g_pre"])
    d = dr + rho_r * (e - rh * torch.mean(e * rh, dim=1, keepdim=True))
    dscale = torch.sum((d * wd).double(), dim=(0, 2)).float()
    dw = col(s["scale"]) * d
    if D is not None:
        dw = dw * D
    dz = dg_post = None
    dmn = dw
    if z is not None:
        dz = (dw * mn * _act_grad(z, c["gate"])).to(dt).reshape(shape)
        dmn = dw * _act(z, c["gate"])
    dm = dmn
    if c["post"]:
        dg_post = torch.sum((dmn * mh).double(), dim=(0, 2)).float()
        f = dmn * col(s["g_post"])
        dm = rho_m * (f - mh * torch.mean(f * mh, dim=1, keepdim=True))
    return _block_outputs(*out, d.to(dt).reshape(shape), dm.to(dt).reshape(shape), dz, dg_post, dscale, dg_pre)


def run(s):
    if own:
        return _run_own(s)
    if s["case"]["op"] == "recurrence":
        return _plain_recurrence(s)
    if s["case"]["op"] == "block":
        return _plain_block(s)
    x = s["x"]
    return (x.float() * _drop_factor(x, s["case"]["p"], s["rng"])).to(x.dtype)


def work(case):
    """Every input read once, every output written once."""
    es = 4 if case["dtype"] == "f32" else 2
    rows = case["B"] * case["C"]
    n = rows * math.prod(_dims(case))
    kind = case["kind"]
    if kind == "step":
        return {"bytes": 5 * n * es + 8 * rows, "flops": 6 * n}
    if kind == "scan":                                        # q, k, v, g -> y; state in and out
        return {"bytes": 5 * n * es + 8 * rows, "flops": 6 * n}
    if kind == "scan_train":                                  # q, k, v, g, dy -> y, dq, dk, dv, dg; s0, ds -> s_end, ds0
        return {"bytes": 10 * n * es + 16 * rows, "flops": 18 * n}
    if kind == "dropout":
        return {"bytes": 2 * n * es, "flops": n}
    gate = case["gate"] != "none"
    if kind == "block":                                       # x, m, z -> r, n
        return {"bytes": (4 + gate) * n * es, "flops": 14 * n}
    return {"bytes": (8 + 2 * gate) * n * es, "flops": 45 * n}      # and dr, dn -> dx, dm, dz


# ---- the definitions in 64 bits -------------------------------------------------------------------------------------

def _exact_scan(a, u, s0):
    """The recurrence itself, one position after the other inside spans, the spans' starts one after the other."""
    R, L = a.shape
    n = max(1, math.isqrt(L))
    spans = (L + n - 1) // n
    pad = spans * n - L
    if pad:
        a = torch.cat([a, torch.ones((R, pad), dtype=a.dtype, device=a.device)], dim=1)
        u = torch.cat([u, torch.zeros((R, pad), dtype=u.dtype, device=u.device)], dim=1)
    a, u = a.reshape(R, spans, n), u.reshape(R, spans, n)
    end, prod = torch.zeros_like(a[:, :, 0]), torch.ones_like(a[:, :, 0])
    for t in range(n):
        end = a[:, :, t] * end + u[:, :, t]
        prod = prod * a[:, :, t]
    state, starts = s0, []
    for j in range(spans):
        starts.append(state)
        state = prod[:, j] * state + end[:, j]
    state = torch.stack(starts, dim=1)
    out = torch.empty_like(a)
    for t in range(n):
        state = a[:, :, t] * state + u[:, :, t]
        out[:, :, t] = state
    return out.reshape(R, spans * n)[:, :L]


def _exact_recurrence(s):
    c = s["case"]
    B, C = c["B"], c["C"]
    q, k, v, g = (s[key].double().reshape(B * C, -1) for key in ("q", "k", "v", "g"))
    L = q.shape[1]
    s0 = s["s0"].double().reshape(-1)
    n = torch.full((B,), L, device=q.device) if s["lengths"] is None else s["lengths"].long()
    n = n.repeat_interleave(C)
    dead = torch.arange(L, device=q.device)[None, :] >= n[:, None]
    a = {"value": lambda t: t, "log": torch.exp, "sigmoid": torch.sigmoid}[c["decay"]](g)
    a = a.masked_fill(dead, 1.0)
    S = _exact_scan(a, (k * v).masked_fill(dead, 0.0), s0)
    shape = s["q"].shape
    out = {"y": (q * S).masked_fill(dead, 0.0).reshape(shape), "s_end": S[:, -1].reshape(B, C).clone()}
    if c["kind"] != "scan_train":
        return out
    dy = s["dy"].double().reshape(B * C, -1).masked_fill(dead, 0.0)
    # mu_t = a_t lam_t, from the row's end to its start: lam_t = q_t dy_t + mu_{t+1}
    nxt = torch.ones_like(a)
    nxt[:, :-1] = a[:, 1:]
    lam = torch.flip(_exact_scan(torch.flip(nxt, [1]), torch.flip(q * dy, [1]), s["ds"].double().reshape(-1)), [1])
    prev = torch.empty_like(S)
    prev[:, 0] = s0
    prev[:, 1:] = S[:, :-1]
    slope = {"value": lambda: 1.0, "log": lambda: a, "sigmoid": lambda: torch.sigmoid(g) * torch.sigmoid(-g)}[c["decay"]]()
    out["dq"] = (dy * S).reshape(shape)
    out["dk"] = (lam * v).masked_fill(dead, 0.0).reshape(shape)
    out["dv"] = (lam * k).masked_fill(dead, 0.0).reshape(shape)
    out["dg"] = (lam * prev * slope).masked_fill(dead, 0.0).reshape(shape)
    out["ds0"] = (a[:, 0] * lam[:, 0]).reshape(B, C)
    return out


def _exact_keep(n, p, rng):
    """Which of n elements stay, on the host in unsigned 64-bit arithmetic."""
    seed, step = (int(t) for t in rng.cpu())
    idx = np.arange((n + 7) // 8, dtype=np.uint64)
    lo32, sh = np.uint64(_M32), np.uint64(32)
    ctr = [idx & lo32, idx >> sh, np.full_like(idx, step & _M32), np.zeros_like(idx)]
    key = [seed & _M32, (seed >> 32) & _M32]
    for _ in range(10):
        first, second = ctr[0] * np.uint64(0xD2511F53), ctr[2] * np.uint64(0xCD9E8D57)
        ctr = [(second >> sh) ^ ctr[1] ^ np.uint64(key[0]), second & lo32, (first >> sh) ^ ctr[3] ^ np.uint64(key[1]), first & lo32]
        key = [(key[0] + 0x9E3779B9) & _M32, (key[1] + 0xBB67AE85) & _M32]
    bits = np.empty((idx.size, 8), dtype=np.uint32)
    for j in range(4):
        bits[:, 2 * j], bits[:, 2 * j + 1] = ctr[j] & np.uint64(0xFFFF), ctr[j] >> np.uint64(16)
    return bits.reshape(-1)[:n] >= _threshold(p)


def _exact_factor(like, p, rng):
    thr = _threshold(p)
    keep = torch.from_numpy(_exact_keep(like.numel(), p, rng)).to(like.device).reshape(like.shape)
    return keep.double() * (65536.0 / (65536 - thr))


def _exact_block(s):
    """A token is a column of C numbers; gradients by the chain rule, one factor after the other."""
    c = s["case"]
    B, C = c["B"], c["C"]

    def wide(t):
        return None if t is None else t.double().reshape(B, C, -1)

    x, m, z = wide(s["x"]), wide(s["m"]), wide(s["z"])
    g_post, scale, g_pre = (None if t is None else t.double().reshape(1, C, 1) for t in (s["g_post"], s["scale"], s["g_pre"]))
    root = lambda t: torch.sqrt((t ** 2).sum(1, keepdim=True) / C + _EPS)
    norm_m = root(m) if c["post"] else None
    b = m / norm_m * g_post if c["post"] else m
    gate = None if z is None else torch.sigmoid(z) * (z if c["gate"] == "silu" else 1.0)
    branch = b if gate is None else b * gate
    f = _exact_factor(x, c["p"], s["rng"]) if c["p"] else None
    if f is not None:
        branch = branch * f
    r = x + scale * branch
    norm_r = root(r)
    shape = s["x"].shape
    r_out, n_out = r.reshape(shape), (r / norm_r * g_pre).reshape(shape)
    if c["kind"] == "block":
        return {"r": r_out, "n": n_out}
    dr, dn = wide(s["dr"]), wide(s["dn"])

    def norm_backward(value, norm, gradient):
        # d(value / norm): gradient / norm - value (value . gradient) / (C norm^3)
        return gradient / norm - value * (value * gradient).sum(1, keepdim=True) / (C * norm ** 3)

    total = dr + norm_backward(r, norm_r, dn * g_pre)
    dbranch = total * scale
    if f is not None:
        dbranch = dbranch * f
    dz = None
    db = dbranch
    if z is not None:
        sg = torch.sigmoid(z)
        slope = sg * (1 - sg) * z + sg if c["gate"] == "silu" else sg * torch.sigmoid(-z)
        dz, db = (dbranch * b * slope).reshape(shape), dbranch * gate
    dg_post, dm = None, db
    if c["post"]:
        dg_post = (db * m / norm_m).sum((0, 2))
        dm = norm_backward(m, norm_m, db * g_post)
    return _block_outputs(r_out, n_out, total.reshape(shape), dm.reshape(shape), dz, dg_post, (total * branch).sum((0, 2)),
                          (dn * r / norm_r).sum((0, 2)))


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "recurrence":
        return _exact_recurrence(s)
    if case["op"] == "block":
        return _exact_block(s)
    return s["x"].double() * _exact_factor(s["x"], case["p"], s["rng"])
