"""Timed cases of the operators of a block's feed-forward half around the
stage-boundary codec, and of its weights' update: norms before and after a block
with its gate and residual scale, the gated feed-forward block, orthogonalised
updates.

Kinds (a case's "kind"):

  block_norm       the end of a block and the start of the next: the block
                   output's norm, its gate, the scaled residual, the next norm
  block_norm_grad  its backward: gradients of output, residual, gains and gate
  gated_ff         act(X Wg) * (X Wu), with the two products where a backward
                   pass will want them ("save")
  gated_ff_grad    its backward: gradients of the input and both weights
  orthogonalize    matrices with the singular values taken towards 1 by five
                   Newton-Schulz steps
  muon             momentum, orthogonalised update and decay of weights in place

Widths, token counts and feed-forward sizes are those of synth.CONFIGS and of the
codec's timed cases (d = 256 .. 8192, ff = 8/3 d .. 4 d, 1 to 32768 tokens).
"""
from __future__ import annotations

import math

import torch

DEV = "cuda"
own = False
EPS = 1e-6
A, B, C = 3.4445, -4.7750, 2.0315  # the Newton-Schulz step's coefficients
STEPS = 5
LR, MOMENTUM, DECAY = 0.02, 0.95, 1e-4


# ---------------------------------------------------------------------------
# cases
# ---------------------------------------------------------------------------
def _norm(kind, dtype, n, d, post=True, gate="none", fn="none", alpha=1.0):
    """gate: "none", "row" (one row of gains for all tokens) or "token"."""
    return {"kind": kind, "dtype": dtype, "n": n, "d": d, "post": post, "gate": gate, "fn": fn,
            "alpha": alpha}


def _ff(kind, dtype, n, d, ff, act="silu", save=False):
    return {"kind": kind, "dtype": dtype, "n": n, "d": d, "ff": ff, "act": act, "save": save}


def _mats(kind, dtype, rows, cols, count):
    return {"kind": kind, "dtype": dtype, "rows": rows, "cols": cols, "count": count}


def listed():
    return [
        # one token of one sequence in serving: the end of a block
        dict(_norm("block_norm", "bf16", 1, 4096, gate="row"), name="block-norm-one-token"),
        # every block's end at the benchmark's 8 x 4096 tokens
        dict(_norm("block_norm", "bf16", 32768, 4096, gate="row", alpha=0.7071), name="block-norm-d4096"),
        # an awkward width, an odd number of tokens, a gate for each token and column
        dict(_norm("block_norm_grad", "bf16", 4999, 1600, gate="token", fn="sigmoid"),
             name="block-norm-grad-d1600"),
        # the backward at the widest model
        dict(_norm("block_norm_grad", "bf16", 16383, 8192, gate="row"), name="block-norm-grad-d8192"),
        # decoding one token: the weights' reading is all there is
        dict(_ff("gated_ff", "bf16", 1, 4096, 14336), name="ff-one-token"),
        # decoding a few dozen sequences together
        dict(_ff("gated_ff", "bf16", 48, 4096, 14336), name="ff-48-tokens"),
        # training at the benchmark's 8 x 4096 tokens, both products kept
        dict(_ff("gated_ff", "bf16", 32768, 4096, 14336, save=True), name="ff-d4096"),
        # odd sizes throughout (rows start at odd offsets), in training
        dict(_ff("gated_ff_grad", "bf16", 4999, 1600, 4267, act="gelu"), name="ff-grad-d1600"),
        # a small float32 model's backward
        dict(_ff("gated_ff_grad", "f32", 2048, 1024, 4096, act="relu"), name="ff-grad-f32"),
        # the smallest program's six square float32 weights
        dict(_mats("orthogonalize", "f32", 256, 256, 6), name="orthogonalize-tiny"),
        # a layer's attention weights at width 4096
        dict(_mats("muon", "bf16", 4096, 4096, 4), name="muon-4096"),
        # down projections of odd widths, stored [out, in]
        dict(_mats("muon", "f32", 1600, 4267, 2), name="muon-1600x4267"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _cost(case):
    w = work(case)
    return w["bytes"] / 5e12 + w["flops"] / 1e14


def draw(rng):
    most = max(_cost(c) for c in listed())
    while True:
        case = _draw(rng)
        if _cost(case) <= most:
            return case


def _draw(rng):
    op = rng.choice(["norm", "ff", "ff", "mats"])
    dtype = "f32" if rng.random() < 0.3 else "bf16"
    if op == "norm":
        d = 256 * _log_int(rng, 1, 32) if rng.random() < 0.6 else _log_int(rng, 200, 8192)
        gate = rng.choice(["none", "row", "token"])
        return _norm(rng.choice(["block_norm", "block_norm_grad"]), dtype, _log_int(rng, 1, 32768), d,
                     post=rng.random() < 0.8, gate=gate,
                     fn="none" if gate == "none" else rng.choice(["none", "sigmoid"]),
                     alpha=rng.choice([1.0, 0.5, 0.7071, 1.25]))
    if op == "ff":
        d = 256 * _log_int(rng, 1, 16) if rng.random() < 0.6 else _log_int(rng, 200, 4096)
        ff = rng.choice([4 * d, 8 * d // 3, int(3.5 * d)])
        kind = rng.choice(["gated_ff", "gated_ff", "gated_ff_grad"])
        return _ff(kind, dtype, _log_int(rng, 1 if kind == "gated_ff" else 64, 32768), d, ff,
                   act=rng.choice(["silu", "silu", "gelu", "relu"]),
                   save=kind == "gated_ff" and rng.random() < 0.4)
    d = 64 * _log_int(rng, 1, 64) if rng.random() < 0.6 else _log_int(rng, 60, 4096)
    ff = rng.choice([d, d, 4 * d, 8 * d // 3])
    r, c = (d, ff) if rng.random() < 0.5 else (ff, d)
    return _mats(rng.choice(["orthogonalize", "muon"]), dtype, r, c, _log_int(rng, 1, 12))


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------
def _type(case):
    return torch.float32 if case["dtype"] == "f32" else torch.bfloat16


def _gen(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(1000003 * int(seed) + sum(ord(c) for c in case["kind"]) + int(case.get("n", 0)))
    return g


def _randn(g, *shape, dtype, std=1.0, mean=0.0):
    """A random matrix, made in pieces of rows so that its float32 form stays small."""
    out = torch.empty(shape, dtype=dtype, device=DEV)
    rows = out if out.dim() > 1 else out[None]
    step = max(1, (1 << 27) // max(1, rows.shape[1]))
    for r in range(0, rows.shape[0], step):
        part = rows[r:r + step]
        part.copy_(torch.randn(part.shape, generator=g, device=DEV) * std + mean)
    return out


def prepare(case, seed):
    if "post" in case:
        return _norm_state(case, seed)
    return (_ff_state if "ff" in case else _mats_state)(case, seed)


def _norm_state(case, seed):
    g, n, d, t = _gen(case, seed), case["n"], case["d"], _type(case)
    s = {"case": case, "X": _randn(g, n, d, dtype=t, std=0.7), "R": _randn(g, n, d, dtype=t, std=2.0),
         "w": _randn(g, d, dtype=t, std=0.1, mean=1.0), "w_post": None, "gate": None}
    if case["post"]:
        s["w_post"] = _randn(g, d, dtype=t, std=0.1, mean=1.0)
    if case["gate"] == "row":
        s["gate"] = _randn(g, d, dtype=t, std=0.2, mean=0.5)
    elif case["gate"] == "token":
        s["gate"] = _randn(g, n, d, dtype=t)
    if case["kind"] == "block_norm_grad":
        # R stands for the h that the forward call left
        s["dY"], s["dH"] = _randn(g, n, d, dtype=t, std=0.01), _randn(g, n, d, dtype=t, std=0.01)
        s["gw"] = torch.zeros(d, device=DEV)
        s["gw_post"] = torch.zeros(d, device=DEV) if case["post"] else None
        s["dgate"] = torch.zeros(d, device=DEV) if case["gate"] == "row" else None
    return s


def _ff_state(case, seed):
    g, n, d, ff, t = _gen(case, seed), case["n"], case["d"], case["ff"], _type(case)
    s = {"case": case, "X": _randn(g, n, d, dtype=t), "Wg": _randn(g, d, ff, dtype=t, std=d ** -0.5),
         "Wu": _randn(g, d, ff, dtype=t, std=d ** -0.5)}
    if case["kind"] == "gated_ff_grad":
        # the two products that the forward call left, and buffers of their gradients
        s["G"], s["U"] = _randn(g, n, ff, dtype=t), _randn(g, n, ff, dtype=t)
        s["dH"] = _randn(g, n, ff, dtype=t, std=0.01)
        s["dG"], s["dU"] = torch.empty_like(s["G"]), torch.empty_like(s["U"])
    return s


def _mats_state(case, seed):
    g, r, c, t = _gen(case, seed), case["rows"], case["cols"], _type(case)
    s = {"case": case, "G": [], "M": [], "W": []}
    k = max(1, min(r, c) // 8)
    for _ in range(case["count"]):
        # gradients of few strong directions among weak ones
        strong = torch.randn(r, k, generator=g, device=DEV) @ torch.randn(k, c, generator=g, device=DEV)
        s["G"].append(((strong * k ** -0.5 + 0.2 * torch.randn(r, c, generator=g, device=DEV)) * 1e-3).to(t))
        if case["kind"] == "muon":
            s["M"].append(5e-3 * torch.randn(r, c, generator=g, device=DEV))
            s["W"].append(_randn(g, r, c, dtype=t, std=c ** -0.5))
    s["scale"] = math.sqrt(max(1.0, r / c))
    return s


# ---------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------
def run(s):
    return (_run_own if own else _run_plain)(s["case"]["kind"], s["case"], s)


def _run_own(kind, case, s):
    import paper_2506_01260_amd as sn
    if kind == "block_norm":
        Y, H = sn.sn_block_norm(s["X"], s["R"], s["w"], w_post=s["w_post"], post=case["post"],
                                gate=s["gate"], gate_fn=case["fn"], alpha=case["alpha"], eps=EPS)
        return {"Y": Y, "H": H}
    if kind == "block_norm_grad":
        dX, dR, dgate = sn.sn_block_norm_backward(
            s["X"], s["R"], s["dY"], s["w"], w_post=s["w_post"], post=case["post"], gate=s["gate"],
            gate_fn=case["fn"], alpha=case["alpha"], dH=s["dH"], eps=EPS, gw=s["gw"],
            gw_post=s["gw_post"], dgate=s["dgate"])
        return {"dX": dX, "dR": dR, "dgate": dgate, "gw": s["gw"], "gw_post": s["gw_post"]}
    if kind == "gated_ff":
        if not case["save"]:
            return {"H": sn.sn_gated_ff(s["X"], s["Wg"], s["Wu"], act=case["act"])}
        H, G, U = sn.sn_gated_ff(s["X"], s["Wg"], s["Wu"], act=case["act"], save=True)
        return {"H": H, "G": G, "U": U}
    if kind == "gated_ff_grad":
        dX, gWg, gWu = sn.sn_gated_ff_backward(s["X"], s["Wg"], s["Wu"], s["G"], s["U"], s["dH"],
                                               act=case["act"], dG=s["dG"], dU=s["dU"])
        return {"dX": dX, "gWg": gWg, "gWu": gWu}
    if kind == "orthogonalize":
        return {"O": sn.sn_orthogonalize(s["G"], steps=STEPS)}
    sn.sn_muon_step(s["W"], s["G"], s["M"], LR, momentum=MOMENTUM, nesterov=True, weight_decay=DECAY,
                    scale=s["scale"], steps=STEPS)
    return {"W": s["W"], "M": s["M"]}


def _run_plain(kind, case, s):
    if kind == "block_norm":
        return _plain_norm(case, s)
    if kind == "block_norm_grad":
        return _plain_norm_grad(case, s)
    if kind == "gated_ff":
        return _plain_ff(case, s)
    if kind == "gated_ff_grad":
        return _plain_ff_grad(case, s)
    return _plain_mats(kind, s)


def _gate(case, s):
    """The gate's values (None without one) and their derivative."""
    if s["gate"] is None:
        return None, None
    g = s["gate"].float()
    if case["fn"] == "none":
        return g, torch.ones_like(g)
    g = 1.0 / (1.0 + torch.exp(-g))
    return g, g * (1.0 - g)


def _inv_rms(h):
    return torch.rsqrt(h.square().mean(1, keepdim=True) + EPS)


def _plain_norm(case, s):
    t = s["X"].dtype
    z = s["X"].float()
    if case["post"]:
        z = z * _inv_rms(z) * s["w_post"].float()
    g, _ = _gate(case, s)
    h = s["R"].float() * case["alpha"] + (z if g is None else g * z)
    return {"Y": (h * _inv_rms(h) * s["w"].float()).to(t), "H": h.to(t)}


def _plain_norm_grad(case, s):
    t = s["X"].dtype
    x, h, dy = s["X"].float(), s["R"].float(), s["dY"].float()
    r = _inv_rms(h)
    u = dy * s["w"].float()
    dh = r * u - h * (r * r * r * (u * h).mean(1, keepdim=True)) + s["dH"].float()
    s["gw"] += (dy * h * r).sum(0)
    g, slope = _gate(case, s)
    q = _inv_rms(x) if case["post"] else None
    z = x * q * s["w_post"].float() if case["post"] else x
    dz = dh if g is None else dh * g
    dgate = None
    if g is not None:
        dgate = dh * z * slope
        if case["gate"] == "row":
            s["dgate"] += dgate.sum(0)
            dgate = s["dgate"]
        else:
            dgate = dgate.to(t)
    dx = dz
    if case["post"]:
        s["gw_post"] += (dz * x * q).sum(0)
        v = dz * s["w_post"].float()
        dx = q * v - x * (q * q * q * (v * x).mean(1, keepdim=True))
    return {"dX": dx.to(t), "dR": (dh * case["alpha"]).to(t), "dgate": dgate, "gw": s["gw"],
            "gw_post": s["gw_post"]}


def _act(name, g):
    """The activation of g and its derivative."""
    if name == "relu":
        on = (g > 0).to(g.dtype)
        return g * on, on
    if name == "silu":
        p = 1.0 / (1.0 + torch.exp(-g))
        return g * p, p * (1.0 + g * (1.0 - p))
    p = 0.5 * (1.0 + torch.erf(g * math.sqrt(0.5)))
    return g * p, p + g * torch.exp(-0.5 * g * g) * (1.0 / math.sqrt(2.0 * math.pi))


def _plain_ff(case, s):
    t, x = s["X"].dtype, s["X"].float()
    G, U = x @ s["Wg"].float(), x @ s["Wu"].float()
    out = {"H": (_act(case["act"], G)[0] * U).to(t)}
    if case["save"]:
        out["G"], out["U"] = G.to(t), U.to(t)
    return out


def _plain_ff_grad(case, s):
    t, x, dh = s["X"].dtype, s["X"].float(), s["dH"].float()
    a, slope = _act(case["act"], s["G"].float())
    dg, du = dh * s["U"].float() * slope, dh * a
    dx = dg @ s["Wg"].float().t() + du @ s["Wu"].float().t()
    return {"dX": dx.to(t), "gWg": (x.t() @ dg).to(t), "gWu": (x.t() @ du).to(t)}


def _plain_orthogonal(m):
    """Singular values towards 1: five steps X <- a X + (b X X^T + c (X X^T)^2) X."""
    norm = torch.sqrt(m.double().square().sum()).float()
    x = m / torch.where(norm > 0, norm, torch.ones_like(norm))
    if m.shape[0] > m.shape[1]:
        x = x.t()
    for _ in range(STEPS):
        p = x @ x.t()
        x = A * x + (B * p + C * (p @ p)) @ x
    return x.t() if m.shape[0] > m.shape[1] else x


def _plain_mats(kind, s):
    if kind == "orthogonalize":
        return {"O": [_plain_orthogonal(g.float()).to(g.dtype) for g in s["G"]]}
    for w, g, m in zip(s["W"], s["G"], s["M"]):
        m.mul_(MOMENTUM).add_(g.float())
        o = _plain_orthogonal(g.float() + MOMENTUM * m)
        w.copy_(w.float() - LR * s["scale"] * o - DECAY * w.float())
    return {"W": s["W"], "M": s["M"]}


# ---------------------------------------------------------------------------
# what a pass cannot do without
# ---------------------------------------------------------------------------
def work(case):
    es = 4 if case["dtype"] == "f32" else 2
    if "post" in case:
        n, d, tok = case["n"], case["d"], 1 if case["gate"] == "token" else 0
        rows = d * (es * (1 + case["post"]) + (es if case["gate"] == "row" else 0))
        if case["kind"] == "block_norm":
            return {"bytes": n * d * es * (4 + tok) + rows, "flops": 14 * n * d}
        return {"bytes": n * d * es * (6 + 2 * tok) + 3 * rows, "flops": 30 * n * d}
    if "ff" in case:
        n, d, ff = case["n"], case["d"], case["ff"]
        if case["kind"] == "gated_ff":
            return {"bytes": es * (n * d + 2 * d * ff + n * ff * (3 if case["save"] else 1)),
                    "flops": 4 * n * d * ff}
        return {"bytes": es * (2 * n * d + 4 * d * ff + 3 * n * ff), "flops": 8 * n * d * ff}
    r, c, k = case["rows"], case["cols"], case["count"]
    m, n = min(r, c), max(r, c)
    # X X^T and its square are symmetric: half the products
    flops = STEPS * (m * (m + 1) * n + m * m * (m + 1) + 2 * m * m * n)
    return {"bytes": k * r * c * (2 * es if case["kind"] == "orthogonalize" else 3 * es + 8),
            "flops": k * flops}


# ---------------------------------------------------------------------------
# the definitions in 64 bits
# ---------------------------------------------------------------------------
def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "block_norm":
        return _join([_exact_norm(case, s, b) for b in _rows(case["n"], case["d"])])
    if case["kind"] == "block_norm_grad":
        return _exact_norm_grad(case, s)
    if case["kind"] == "gated_ff":
        wg, wu = s["Wg"].double(), s["Wu"].double()
        return _join([_exact_ff(case, s, b, wg, wu) for b in _rows(case["n"], case["ff"])])
    if case["kind"] == "gated_ff_grad":
        return _exact_ff_grad(case, s)
    return _exact_mats(case, s)


def _rows(n, width):
    step = max(1, (1 << 26) // width)
    return [slice(r, min(n, r + step)) for r in range(0, n, step)]


def _join(parts):
    return {k: torch.cat([p[k] for p in parts]) for k in parts[0]}


def _unit(x):
    """(x over its root mean square, that root mean square)."""
    rms = (x.pow(2).sum(1, keepdim=True) / x.shape[1] + EPS).sqrt()
    return x / rms, rms


def _exact_gate(case, s, b):
    if s["gate"] is None:
        return torch.ones((), dtype=torch.float64, device=DEV)
    g = (s["gate"][b] if case["gate"] == "token" else s["gate"]).double()
    return torch.sigmoid(g) if case["fn"] == "sigmoid" else g


def _exact_norm(case, s, b):
    x = s["X"][b].double()
    z = _unit(x)[0] * s["w_post"].double() if case["post"] else x
    h = case["alpha"] * s["R"][b].double() + z * _exact_gate(case, s, b)
    return {"Y": _unit(h)[0] * s["w"].double(), "H": h}


def _exact_norm_grad(case, s):
    d, parts = case["d"], []
    sums = {k: torch.zeros(d, dtype=torch.float64, device=DEV) for k in ("gw", "gw_post", "dgate")}
    for b in _rows(case["n"], d):
        dy, (e, rms) = s["dY"][b].double(), _unit(s["R"][b].double())
        sums["gw"] += (dy * e).sum(0)
        v = dy * s["w"].double()
        dh = (v - e * (v * e).sum(1, keepdim=True) / d) / rms + s["dH"][b].double()
        gate, x = _exact_gate(case, s, b), s["X"][b].double()
        unit, xrms = _unit(x)
        z = unit * s["w_post"].double() if case["post"] else x
        slope = gate * (1 - gate) if case["fn"] == "sigmoid" else 1.0
        part = {"dX": dh * gate, "dR": case["alpha"] * dh}
        if case["gate"] == "token":
            part["dgate"] = dh * z * slope
        else:
            sums["dgate"] += (dh * z * slope).sum(0)
        if case["post"]:
            sums["gw_post"] += (part["dX"] * unit).sum(0)
            v = part["dX"] * s["w_post"].double()
            part["dX"] = (v - unit * (v * unit).sum(1, keepdim=True) / d) / xrms
        parts.append(part)
    whole = _join(parts)
    whole["gw"], whole["gw_post"] = sums["gw"], sums["gw_post"] if case["post"] else None
    if case["gate"] != "token":
        whole["dgate"] = sums["dgate"] if case["gate"] == "row" else None
    return whole


def _exact_act(name, g):
    """The activation and its derivative, from torch's own forms in 64 bits."""
    f = {"silu": torch.nn.functional.silu, "gelu": torch.nn.functional.gelu, "relu": torch.relu}[name]
    with torch.enable_grad():
        x = g.detach().requires_grad_(True)
        y = f(x)
        slope, = torch.autograd.grad(y.sum(), x)
    return y.detach(), slope


def _exact_ff(case, s, b, wg, wu):
    x = s["X"][b].double()
    G, U = x @ wg, x @ wu
    part = {"H": _exact_act(case["act"], G)[0] * U}
    if case["save"]:
        part["G"], part["U"] = G, U
    return part


def _exact_ff_grad(case, s):
    wg, wu, dx = s["Wg"].double(), s["Wu"].double(), []
    gwg, gwu = torch.zeros_like(wg), torch.zeros_like(wu)
    for b in _rows(case["n"], case["ff"]):
        x, dh = s["X"][b].double(), s["dH"][b].double()
        a, slope = _exact_act(case["act"], s["G"][b].double())
        dg, du = slope * s["U"][b].double() * dh, a * dh
        dx.append(torch.cat([dg, du], 1) @ torch.cat([wg, wu], 1).t())
        gwg += x.t() @ dg
        gwu += x.t() @ du
    return {"dX": torch.cat(dx), "gWg": gwg, "gWu": gwu}


def _exact_orthogonal(m):
    """The steps' polynomials of the smaller Gram matrix K = X X^T or X^T X, multiplied
    up (they commute), and one product with X at the end."""
    x = m / m.norm() if bool(m.norm() > 0) else m
    tall = m.shape[0] > m.shape[1]
    gram = x.t() @ x if tall else x @ x.t()
    one = torch.eye(gram.shape[0], dtype=torch.float64, device=DEV)
    whole = one
    for _ in range(STEPS):
        q = A * one + gram @ (B * one + C * gram)
        whole, gram = q @ whole, q @ gram @ q
    return x @ whole if tall else whole @ x


def _exact_mats(case, s):
    if case["kind"] == "orthogonalize":
        return {"O": [_exact_orthogonal(g.double()) for g in s["G"]]}
    out = {"W": [], "M": []}
    for w, g, m in zip(s["W"], s["G"], s["M"]):
        m1 = MOMENTUM * m.double() + g.double()
        o = _exact_orthogonal(g.double() + MOMENTUM * m1)
        out["W"].append((1 - DECAY) * w.double() - LR * s["scale"] * o)
        out["M"].append(m1)
    return out
