"""Heads and the delta rule beside the long convolution, as they are measured.

Two operators on the library's layout [B, heads x channels, L_1..L_N], with what each of them computes written out in `run`'s
plain forms (`own` false) and called through the library's entry points where `own` is true:

    delta        the gated delta rule on a matrix state per head,  u_t = beta_t (v_t - a_t S_{t-1} k_t),  S_t = a_t S_{t-1} + u_t k_t^T,
                 y_t = S_t q_t;  kinds: "step" (one token against kept states), "scan" (a sequence, from states to states),
                 "scan_train" (a sequence and its gradients).  Several value heads may share one head of queries and keys
    heads        queries and keys normalised per head and turned by their position on the grid, one rotation per pair of channels,
                 every axis of the grid with pairs of its own; kinds: "turn", "turn_train" (and its gradients)

A case is a dict of plain values.  `exact` evaluates the definitions in 64 bits, token by token.
"""
import math

import torch

own = False

_EPS = 1e-6
_BASE = 10000.0
_SPAN = 64                                     # tokens that the plain form of the delta rule takes together
_DECAYS = ("log", "sigmoid", "none")
_NORMS = ("rms", "l2", "none")


def _delta_case(name, kind, L, B, H, Hk, Dk, Dv, dtype, decay, ragged):
    c = {"op": "delta", "kind": kind, "dims": str(L), "B": B, "H": H, "Hk": Hk, "Dk": Dk, "Dv": Dv, "dtype": dtype, "decay": decay, "ragged": ragged}
    return dict(c, name=name) if name else c


def _heads_case(name, kind, dims, axes, B, Hq, Hk, D, dtype, norm, weights, positions):
    c = {"op": "heads", "kind": kind, "dims": dims, "axes": axes, "B": B, "Hq": Hq, "Hk": Hk, "D": D, "dtype": dtype, "norm": norm,
         "weights": weights, "positions": positions}
    return dict(c, name=name) if name else c


def listed():
    return [
        # one generated token for a batch of 32 sequences, some of which have ended: 768 channels as six heads
        _delta_case("delta_step", "step", 1, 32, 6, 6, 128, 128, "bf16", "log", True),
        # prompts of unequal length, carried on from states: 768 channels as twelve narrow heads
        _delta_case("delta_prompts", "scan", 2000, 16, 12, 12, 64, 64, "bf16", "sigmoid", True),
        # long-context genomics layer, the benchmark's sequence: few heads, a very long axis
        _delta_case("delta_genomics", "scan", 262144, 2, 2, 2, 128, 128, "bf16", "log", False),
        # training step on the benchmark's vision grid read as a sequence
        _delta_case("delta_vision", "scan_train", 4096, 16, 6, 6, 128, 128, "bf16", "log", False),
        # training step of a long-context layer
        _delta_case("delta_long", "scan_train", 32768, 2, 2, 2, 128, 128, "bf16", "log", False),
        # training step on a padded batch, fp32, odd length, heads that share queries and keys, odd head sizes
        _delta_case("delta_padded", "scan_train", 1531, 5, 6, 3, 50, 97, "f32", "sigmoid", True),
        # the token's queries and keys, each sequence at a position of its own
        _heads_case("heads_token", "turn", "1", "64", 32, 6, 6, 128, "bf16", "l2", True, True),
        # inference on the benchmark's vision grid, rows and columns
        _heads_case("heads_vision", "turn", "64x64", "16x16", 16, 12, 12, 64, "bf16", "l2", True, False),
        # training step of the long-context layer
        _heads_case("heads_long", "turn_train", "262144", "64", 2, 2, 2, 128, "bf16", "l2", True, False),
        # training step on an odd grid, keys shared by query heads, part of the channels without a position
        _heads_case("heads_odd", "turn_train", "31x33", "8x10", 8, 4, 2, 50, "bf16", "rms", True, False),
        # training step on volumes, three axes, fp32
        _heads_case("heads_volume", "turn_train", "96x96x96", "11x11x10", 1, 1, 1, 64, "f32", "rms", True, False),
    ]


def _log(rng, lo, hi):
    return math.exp(rng.uniform(math.log(lo), math.log(hi)))


def draw(rng):
    """Sequences of 1 to 65536 positions (the delta rule's gradients: 32768), planes of 4 to 128 and volumes of 4 to 64 per axis,
    heads of 8 to 128 channels, odd extents among them; the batch follows from a budget of elements."""
    kind = rng.choice(["step", "scan", "scan", "scan_train", "scan_train", "turn", "turn_train"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    if kind in ("step", "scan", "scan_train"):
        Dk = rng.choice([64, 128, 128, round(_log(rng, 8, 128))])
        Dv = rng.choice([Dk, Dk, round(_log(rng, 8, 128))])
        decay, ragged = rng.choice(_DECAYS), rng.random() < 0.5
        share = rng.choice([1, 1, 2, 3])
        if kind == "step":
            Hk = round(_log(rng, 1, 8))
            return _delta_case("", kind, 1, round(_log(rng, 1, 64)), Hk * share, Hk, Dk, Dv, dtype, decay, ragged)
        budget = _log(rng, 1 << 12, 1 << 17)                              # tokens x heads
        L = max(1, round(_log(rng, 1, min(65536 if kind == "scan" else 32768, budget))))
        rows = max(1, int(budget / L))
        Hk = max(1, min(8, rows // share))
        return _delta_case("", kind, L, max(1, min(32, rows // (Hk * share))), Hk * share, Hk, Dk, Dv, dtype, decay, ragged)
    budget = _log(rng, 1 << 14, 1 << 24)
    D = 2 * round(_log(rng, 4, 64))
    ndim = rng.choice([1, 1, 2, 2, 3])
    top, low = {1: 65536, 2: 128, 3: 64}[ndim], {1: 1, 2: 4, 3: 4}[ndim]
    base = _log(rng, low, min(top, max(low, (budget / D) ** (1.0 / ndim))))
    dims = [max(low, min(top, round(base * _log(rng, 0.7, 1.4)))) for _ in range(ndim)]
    each = D // 2 // ndim
    axes = [each if rng.random() < 0.7 else max(1, each // 2) for _ in range(ndim)]
    heads = max(2, int(budget / D / math.prod(dims)))
    Hk = max(1, min(8, heads // 2))
    Hq = Hk * rng.choice([1, 1, 2])
    return _heads_case("", kind, "x".join(map(str, dims)), "x".join(map(str, axes)), max(1, min(32, heads // (Hq + Hk))), Hq, Hk, D, dtype,
                       rng.choice(_NORMS), rng.random() < 0.7, rng.random() < 0.3)


def _ints(text):
    return tuple(int(d) for d in text.split("x"))


def _torch_dtype(case):
    return torch.float32 if case["dtype"] == "f32" else torch.bfloat16


def prepare(case, seed):
    dev = "cuda"
    gen = torch.Generator(device=dev)
    gen.manual_seed(seed * 1000003 + 31)
    dt, dims, B = _torch_dtype(case), _ints(case["dims"]), case["B"]

    def normal(*sh, dtype=torch.float32):
        return torch.randn(sh, generator=gen, device=dev).to(dtype)

    def uniform(sh, lo, hi):
        return torch.rand(sh, generator=gen, device=dev) * (hi - lo) + lo

    s = {"case": case}
    if case["op"] == "heads":
        Hq, Hk, D = case["Hq"], case["Hk"], case["D"]
        s["q"], s["k"] = normal(B, Hq * D, *dims, dtype=dt), normal(B, Hk * D, *dims, dtype=dt)
        s["g_q"] = 1.0 + 0.1 * normal(D) if case["weights"] else None
        s["g_k"] = 1.0 + 0.1 * normal(D) if case["weights"] else None
        s["positions"] = None
        if case["positions"]:                                             # every sequence somewhere in its own long context
            start = torch.floor(uniform((B, len(dims)) + (1,) * len(dims), 0, 100000)).to(torch.int32)
            s["positions"] = (start + _grid(dims, dev)[None]).to(torch.int32).contiguous()
        if case["kind"] == "turn_train":
            s["dq"], s["dk"] = normal(B, Hq * D, *dims, dtype=dt), normal(B, Hk * D, *dims, dtype=dt)
        return s
    L, H, Hk, Dk, Dv = dims[0], case["H"], case["Hk"], case["Dk"], case["Dv"]

    def unit():                                                           # as a head's norm leaves queries and keys
        t = normal(B, Hk, Dk, L)
        return (t / torch.sqrt((t * t).sum(2, keepdim=True) + _EPS)).reshape(B, Hk * Dk, L).to(dt)

    s["q"], s["k"] = unit(), unit()
    s["v"] = normal(B, H * Dv, L, dtype=dt)
    s["beta"] = 1.0 / (1.0 + torch.exp(-normal(B, H, L)))
    # a memory of its own for every head, from a few tokens to thousands, modulated by every token
    if case["decay"] == "log":
        s["g"] = -torch.exp(uniform((1, H, 1), math.log(1e-3), math.log(1.0))) * torch.log1p(torch.exp(normal(B, H, L)))
    else:
        s["g"] = uniform((1, H, 1), 0.0, 6.0) + normal(B, H, L) if case["decay"] == "sigmoid" else None
    s["s0"] = 0.3 * normal(B, H, Dv, Dk)
    s["lengths"] = None
    if case["ragged"]:
        n = torch.floor(uniform((B,), 0.4, 1.0) * (L + 1)) if L > 1 else (uniform((B,), 0.0, 1.0) < 0.9).float()
        s["lengths"] = n.clamp(0, L).to(torch.int32)
    if case["kind"] == "step":
        for key in ("q", "k", "v", "g", "beta"):
            s[key] = s[key].squeeze(-1).contiguous() if s[key] is not None else None
    if case["kind"] == "scan_train":
        s["dy"] = normal(B, H * Dv, L, dtype=dt)
        s["ds"] = 0.3 * normal(B, H, Dv, Dk)
    return s


# ---- the framework's calls -----------------------------------------------------------------------------------------

def _op(s):
    """The object a program keeps: made once, on the first pass."""
    if "own_op" not in s:
        from paper_2607_19378_b200 import hyenand as hn
        c = s["case"]
        if c["op"] == "heads":
            s["own_op"] = hn.Heads(_ints(c["dims"]), c["B"], c["Hq"], c["Hk"], c["D"], dtype=_torch_dtype(c), norm=c["norm"], axes=_ints(c["axes"]),
                                   base=_BASE, eps=_EPS)
        else:
            s["own_op"] = hn.DeltaRule(_ints(c["dims"])[0], c["B"], c["H"], c["Dk"], c["Dv"], Hk=c["Hk"], decay=c["decay"], dtype=_torch_dtype(c))
        if c["kind"] == "step":
            s["state"] = torch.empty_like(s["s0"])                        # the states before and after a token, kept side by side
    return s["own_op"]


def _run_own(s):
    c, op = s["case"], _op(s)
    if c["op"] == "heads":
        weights = {"g_q": s["g_q"], "g_k": s["g_k"], "positions": s["positions"]}
        q, k = op.forward(s["q"], s["k"], **weights)
        if c["kind"] == "turn":
            return {"q": q, "k": k}
        return _heads_outputs(q, k, *op.backward(s["q"], s["k"], s["dq"], s["dk"], **weights))
    x = (s["q"], s["k"], s["v"], s["g"], s["beta"])
    if c["kind"] == "step":
        return {"y": op.step(*x, s["s0"], new_state=s["state"], active=s["lengths"]), "s_end": s["state"]}
    if c["kind"] == "scan":
        y, s_end = op.forward(*x, s0=s["s0"], lengths=s["lengths"])
        return {"y": y, "s_end": s_end}
    y, s_end, marks = op.forward(*x, s0=s["s0"], lengths=s["lengths"], marks=True)
    return _delta_outputs(y, s_end, *op.backward(*x, marks, s["dy"], ds_end=s["ds"], lengths=s["lengths"]))


def _heads_outputs(q, k, dq, dk, dg_q, dg_k):
    out = {"q": q, "k": k, "dq": dq, "dk": dk}
    return out if dg_q is None else dict(out, dg_q=dg_q, dg_k=dg_k)


def _delta_outputs(y, s_end, dq, dk, dv, dg, dbeta, ds0):
    out = {"y": y, "s_end": s_end, "dq": dq, "dk": dk, "dv": dv, "dbeta": dbeta, "ds0": ds0}
    return out if dg is None else dict(out, dg=dg)


# ---- plain forms ---------------------------------------------------------------------------------------------------

def _grid(dims, device):
    """The positions of a grid's tokens, one plane per axis."""
    planes = torch.meshgrid(*(torch.arange(n, device=device) for n in dims), indexing="ij")
    return torch.stack(planes)


def _angles(s):
    """[1 or B, pairs, T], of the pairs that are turned, in 64 bits: a far position leaves nothing of an angle in 32."""
    c = s["case"]
    dims, axes = _ints(c["dims"]), _ints(c["axes"])
    pos = _grid(dims, s["q"].device)[None] if s["positions"] is None else s["positions"]
    pos = pos.reshape(pos.shape[0], len(dims), -1).double()
    rows = []
    for n, pairs in enumerate(axes):
        freq = _BASE ** (-torch.arange(pairs, device=pos.device, dtype=torch.float64) / pairs)
        rows.append(pos[:, n, None, :] * freq[None, :, None])
    return torch.cat(rows, dim=1)


def _turn(x, cos, sin):
    """Pairs (i, i + D/2) of [B, H, D, T]; cos and sin of the first pairs, the others stay."""
    half, m = x.shape[2] // 2, cos.shape[2]
    a, b = x[:, :, :m], x[:, :, half:half + m]
    out = x.clone()
    out[:, :, :m] = a * cos - b * sin
    out[:, :, half:half + m] = a * sin + b * cos
    return out


def _plain_heads(s):
    c = s["case"]
    dt, D, B = _torch_dtype(c), c["D"], c["B"]
    angle = _angles(s)[:, None]
    cos, sin = torch.cos(angle).float(), torch.sin(angle).float()
    out = {}
    for key, H in (("q", c["Hq"]), ("k", c["Hk"])):
        x = s[key].float().reshape(B, H, D, -1)
        w = torch.ones(D, device=x.device) if s["g_" + key] is None else s["g_" + key]
        w = w[None, None, :, None]
        rho = None
        if c["norm"] != "none":
            total = torch.sum(x * x, dim=2, keepdim=True)
            rho = torch.rsqrt((total / D if c["norm"] == "rms" else total) + _EPS)
        hat = x * rho if rho is not None else x
        out[key] = _turn(hat * w, cos, sin).to(dt).reshape(s[key].shape)
        if c["kind"] == "turn":
            continue
        dn = _turn(s["d" + key].float().reshape(B, H, D, -1), cos, -sin)
        if s["g_" + key] is not None:
            out["dg_" + key] = torch.sum((dn * hat).double(), dim=(0, 1, 3)).float()
        e = dn * w
        if rho is not None:
            dot = torch.sum(e * hat, dim=2, keepdim=True)
            e = rho * (e - hat * (dot / D if c["norm"] == "rms" else dot))
        out["d" + key] = e.to(dt).reshape(s[key].shape)
    return out if c["kind"] == "turn" else _heads_outputs(out["q"], out["k"], out["dq"], out["dk"], out.get("dg_q"), out.get("dg_k"))


def _rows(t, heads, share):
    """[B, heads x D, L] -> [B H, L, D] in 32 bits, shared heads repeated."""
    B, C, L = t.shape
    t = t.float().reshape(B, heads, 1, C // heads, L).expand(B, heads, share, C // heads, L)
    return t.reshape(B * heads * share, C // heads, L).transpose(1, 2)


def _plain_delta(s):
    c = s["case"]
    dt, B, H, Hk, Dk, Dv = _torch_dtype(c), c["B"], c["H"], c["Hk"], c["Dk"], c["Dv"]
    step, share = c["kind"] == "step", H // Hk
    wide = lambda t: t.unsqueeze(-1) if step else t
    q, k, v = _rows(wide(s["q"]), Hk, share), _rows(wide(s["k"]), Hk, share), _rows(wide(s["v"]), H, 1)
    R, L = q.shape[0], q.shape[1]
    beta = wide(s["beta"]).reshape(R, L)
    graw = wide(s["g"]).reshape(R, L) if s["g"] is not None else torch.zeros_like(beta)
    g = -torch.log1p(torch.exp(-graw)) if c["decay"] == "sigmoid" else graw
    live = torch.ones((R, L), dtype=torch.bool, device=q.device)
    if s["lengths"] is not None:
        live = (torch.arange(L, device=q.device)[None, :] < s["lengths"][:, None]).repeat_interleave(H, dim=0)
    zero = lambda t: torch.where(live.unsqueeze(-1), t, 0.0)
    q, k, v = zero(q), zero(k), zero(v)
    beta, g = torch.where(live, beta, 0.0), torch.where(live, g, 0.0)
    N = _SPAN
    chunks = (L + N - 1) // N
    cut = lambda t: torch.nn.functional.pad(t, (0, 0) * (t.dim() - 2) + (0, chunks * N - L)).reshape((R, chunks, N) + t.shape[2:])
    q, k, v, beta, g = cut(q), cut(k), cut(v), cut(beta), cut(g)
    G = torch.cumsum(g.double(), dim=2)                                   # far sums next to small differences
    lower = torch.tril(torch.ones((N, N), dtype=torch.bool, device=q.device))
    ratio = torch.where(lower, torch.exp(torch.where(lower, G[..., :, None] - G[..., None, :], 0.0)), 0.0).float()
    gam, rest, last = torch.exp(G).float()[..., None], torch.exp(G[..., -1:] - G).float()[..., None], torch.exp(G[..., -1]).float()[..., None, None]
    kk = torch.tril(ratio * (k @ k.mT), -1)
    T = beta[..., None] * kk
    A = torch.zeros_like(T)
    for i in range(N):                                                    # (I + T) A = I, row after row
        A[..., i, :] = -(T[..., i:i + 1, :] @ A)[..., 0, :]
        A[..., i, i] += 1.0
    P = ratio * (q @ k.mT)
    bet = beta[..., None]
    S, before, U, left = s["s0"].reshape(R, Dv, Dk), [], [], []
    for n in range(chunks):
        before.append(S)
        r = v[:, n] - gam[:, n] * (k[:, n] @ S.mT)
        u = A[:, n] @ (bet[:, n] * r)
        left.append(r)
        U.append(u)
        S = last[:, n] * S + (rest[:, n] * u).mT @ k[:, n]
    S0, U, left = torch.stack(before, 1), torch.stack(U, 1), torch.stack(left, 1)
    y = gam * (q @ S0.mT) + P @ U

    def back(t, heads, D, dtype):                                         # [R, chunks, N, D] -> [B, heads x D, L]
        t = t.reshape(R, chunks * N, D)[:, :L].mT.reshape(B, heads, R // B // heads, D, L).sum(2)
        return t.reshape(B, heads * D, L).to(dtype)

    out = {"y": back(y, H, Dv, dt), "s_end": S.reshape(B, H, Dv, Dk).clone()}
    if step:
        out["y"] = out["y"].squeeze(-1)
    if c["kind"] != "scan_train":
        return out
    dy = cut(zero(_rows(s["dy"], H, 1)))
    Pdy = P.mT @ dy
    dS, after, dZ = s["ds"].reshape(R, Dv, Dk), [], []
    for n in reversed(range(chunks)):
        after.append(dS)
        dz = A[:, n].mT @ (Pdy[:, n] + rest[:, n] * (k[:, n] @ dS.mT))
        dZ.append(dz)
        dS = last[:, n] * dS + (gam[:, n] * dy[:, n]).mT @ q[:, n] - (gam[:, n] * bet[:, n] * dz).mT @ k[:, n]
    dS1, dZ = torch.stack(after[::-1], 1), torch.stack(dZ[::-1], 1)
    dR = bet * dZ
    F = ratio * (dy @ U.mT)
    W = dZ @ U.mT
    E = -bet * ratio * torch.tril(W, -1)
    dq = gam * (dy @ S0) + F @ k
    dke = E @ k - gam * (dR @ S0)
    dkw = F.mT @ q + E.mT @ k + rest * (U @ dS1)
    S1 = torch.cat([S0[:, 1:], S[:, None]], dim=1)
    dG = torch.sum((q * dq + k * dke - k * dkw).double(), dim=-1)
    dG[..., -1] += torch.sum((S1 * dS1).double(), dim=(-1, -2))
    dg = torch.flip(torch.cumsum(torch.flip(dG, [2]), dim=2), [2]).float()
    if c["decay"] == "sigmoid":
        dg = dg / (1.0 + torch.exp(cut(graw)))
    dbeta = torch.sum((dZ * left).double(), dim=-1) - torch.sum((W * kk).double(), dim=-1)
    rows = lambda t: torch.where(live, t.reshape(R, chunks * N)[:, :L].float(), 0.0).reshape(B, H, L)
    return _delta_outputs(out["y"], out["s_end"], back(dq, Hk, Dk, dt), back(dke + dkw, Hk, Dk, dt), back(dR, H, Dv, dt),
                          rows(dg) if s["g"] is not None else None, rows(dbeta), dS.reshape(B, H, Dv, Dk))


def run(s):
    if own:
        return _run_own(s)
    return _plain_heads(s) if s["case"]["op"] == "heads" else _plain_delta(s)


def work(case):
    """Every input read once, every output written once; the delta rule's products as the token by token form has them."""
    es = 4 if case["dtype"] == "f32" else 2
    n = case["B"] * math.prod(_ints(case["dims"]))
    if case["op"] == "heads":
        elements = n * (case["Hq"] + case["Hk"]) * case["D"]
        extra = 4 * n * len(_ints(case["dims"])) if case["positions"] else 0
        if case["kind"] == "turn":
            return {"bytes": 2 * elements * es + extra, "flops": 7 * elements}
        return {"bytes": 4 * elements * es + elements * es + extra, "flops": 24 * elements}        # q, k, dq', dk' -> q', k', dq, dk
    H, Hk, Dk, Dv = case["H"], case["Hk"], case["Dk"], case["Dv"]
    states = case["B"] * H * Dk * Dv
    gates = n * H * 4 * (1 if case["decay"] == "none" else 2)
    flops = 6 * n * H * Dk * Dv
    if case["kind"] != "scan_train":                                      # q, k, v, g, beta, s0 -> y, s_end
        return {"bytes": 2 * n * (Hk * Dk + H * Dv) * es + gates + 8 * states, "flops": flops}
    # and dy, ds -> dq, dk, dv, dg, dbeta, ds0
    return {"bytes": n * (4 * Hk * Dk + 4 * H * Dv) * es + 2 * gates + 16 * states, "flops": 4 * flops}


# ---- the definitions in 64 bits -------------------------------------------------------------------------------------

def _exact_heads(s):
    """Pairs as complex numbers, the gradient of the norm by the chain rule."""
    c = s["case"]
    B, D, dims, axes = c["B"], c["D"], _ints(c["dims"]), _ints(c["axes"])
    where = _grid(dims, s["q"].device).unsqueeze(0) if s["positions"] is None else s["positions"]
    where = where.reshape(where.shape[0], len(dims), -1)
    turns = torch.zeros((where.shape[0], D // 2, where.shape[2]), dtype=torch.float64, device=where.device)
    row = 0
    for n, pairs in enumerate(axes):
        for j in range(pairs):
            turns[:, row] = where[:, n].double() * math.pow(_BASE, -j / pairs)
            row += 1
    unit = torch.polar(torch.ones_like(turns), turns)[:, None]

    def turned(x, by):
        z = torch.complex(x[:, :, :D // 2], x[:, :, D // 2:]) * by
        return torch.cat([z.real, z.imag], dim=2)

    out = {}
    for key, H in (("q", c["Hq"]), ("k", c["Hk"])):
        x = s[key].double().reshape(B, H, D, -1)
        g = s["g_" + key]
        g = torch.ones(D, dtype=torch.float64, device=x.device) if g is None else g.double()
        g = g.reshape(1, 1, D, 1)
        count = {"rms": D, "l2": 1, "none": 0}[c["norm"]]
        size = torch.sqrt((x ** 2).sum(2, keepdim=True) / count + _EPS) if count else torch.ones_like(x[:, :, :1])
        out[key] = turned(x / size * g, unit).reshape(s[key].shape)
        if c["kind"] == "turn":
            continue
        d = turned(s["d" + key].double().reshape(B, H, D, -1), unit.conj())
        if s["g_" + key] is not None:
            out["dg_" + key] = (d * x / size).sum((0, 1, 3))
        d = d * g
        grad = d / size
        if count:
            grad = grad - x * (x * d).sum(2, keepdim=True) / (count * size ** 3)
        out["d" + key] = grad.reshape(s[key].shape)
    return out if c["kind"] == "turn" else _heads_outputs(out["q"], out["k"], out["dq"], out["dk"], out.get("dg_q"), out.get("dg_k"))


def _exact_delta(s):
    """The rule itself, one token after the other; gradients by the chain rule from the last token to the first, the states of a
    span computed again from its start."""
    c = s["case"]
    B, H, Hk, Dk, Dv = c["B"], c["H"], c["Hk"], c["Dk"], c["Dv"]
    L, R, share = _ints(c["dims"])[0], B * H, H // Hk
    by_token = lambda t, heads, n: t.double().reshape(B, heads, -1, L).repeat_interleave(n, dim=1).reshape(R, -1, L).permute(2, 0, 1).contiguous()
    q, k, v = by_token(s["q"], Hk, share), by_token(s["k"], Hk, share), by_token(s["v"], H, 1)
    beta = s["beta"].double().reshape(R, L).t().contiguous()
    raw = s["g"].double().reshape(R, L).t().contiguous() if s["g"] is not None else None
    a = torch.ones_like(beta) if raw is None else torch.exp(raw) if c["decay"] == "log" else torch.sigmoid(raw)
    live = torch.ones_like(beta)
    if s["lengths"] is not None:
        live = (torch.arange(L, device=q.device)[:, None] < s["lengths"].long().repeat_interleave(H)[None, :]).double()
    beta, a = torch.where(live > 0, beta, 0.0), torch.where(live > 0, a, 1.0)
    q, k, v = q * live[..., None], k * live[..., None], v * live[..., None]
    # tokens as columns, cut apart once
    fades, rates = a[:, :, None, None].unbind(0), beta[:, :, None, None].unbind(0)
    columns, turned, values = k.unsqueeze(-1).unbind(0), k.unsqueeze(-2).unbind(0), v.unsqueeze(-1).unbind(0)

    def token(S, t):
        S = fades[t] * S
        e = torch.baddbmm(values[t], S, columns[t], alpha=-1.0)
        return S, e, torch.baddbmm(S, rates[t] * e, turned[t])

    S = s["s0"].double().reshape(R, Dv, Dk)
    train = c["kind"] == "scan_train"
    span, starts = 32, []
    y = torch.empty_like(v)
    asked, answers = q.unsqueeze(-1).unbind(0), y.unsqueeze(-1).unbind(0)
    for t in range(L):
        if train and t % span == 0:
            starts.append(S)
        S = token(S, t)[2]
        torch.bmm(S, asked[t], out=answers[t])
    lay = lambda t, D: t.permute(1, 2, 0).reshape(B, H * D, L)
    out = {"y": lay(y, Dv)[..., 0] if c["kind"] == "step" else lay(y, Dv), "s_end": S.reshape(B, H, Dv, Dk)}
    if not train:
        return out
    dy = by_token(s["dy"], H, 1) * live[..., None]
    dq, dk, dv, da, db = torch.empty_like(q), torch.empty_like(k), torch.empty_like(v), torch.empty_like(a), torch.empty_like(beta)
    D = s["ds"].double().reshape(R, Dv, Dk)                               # gradient of the state behind token t
    for first in range((L - 1) // span * span, -1, -span):
        kept, S = [], starts.pop()
        for t in range(first, min(first + span, L)):
            faded, e, nxt = token(S, t)
            kept.append((S, faded, e, nxt))
            S = nxt
        for t in range(min(first + span, L) - 1, first - 1, -1):
            S, faded, e, nxt = kept.pop()
            e = e[:, :, 0]
            dq[t] = torch.bmm(dy[t][:, None, :], nxt)[:, 0]
            D = torch.baddbmm(D, dy[t][:, :, None], q[t][:, None, :])
            du = torch.bmm(D, k[t][:, :, None])[:, :, 0]
            de = beta[t][:, None] * du
            db[t] = (du * e).sum(1)
            dv[t] = de
            dk[t] = torch.bmm((beta[t][:, None] * e)[:, None, :], D)[:, 0] - torch.bmm(de[:, None, :], faded)[:, 0]
            D = torch.baddbmm(D, de[:, :, None], k[t][:, None, :], alpha=-1.0)
            da[t] = (D * S).sum((1, 2))
            D = a[t][:, None, None] * D
    dg = None
    if raw is not None:
        dg = da * a if c["decay"] == "log" else da * a * torch.sigmoid(-raw)
        dg = (dg * live).t().reshape(B, H, L)
    join = lambda t: t.permute(1, 2, 0).reshape(B, Hk, share, Dk, L).sum(2).reshape(B, Hk * Dk, L)
    return _delta_outputs(out["y"], out["s_end"], join(dq * live[..., None]), join(dk * live[..., None]), lay(dv, Dv), dg, (db * live).t().reshape(B, H, L),
                          D.reshape(B, H, Dv, Dk))


def exact(case, seed):
    s = prepare(case, seed)
    return _exact_heads(s) if case["op"] == "heads" else _exact_delta(s)
