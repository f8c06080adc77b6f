"""Timed cases of the operators of a training step around the stage-boundary
codec: token log probabilities, root-mean-square norm, gradient clipping.

Kinds (a case's "kind"):

  logprobs       log probabilities of given tokens with entropy and top
                 alternatives, from a matrix of logits (scoring, decoding)
  logprobs_grad  the gradient of the logits for given gradients of the log
                 probabilities and entropies (policy training)
  loss           weighted log probabilities and the logits' gradient in one call
                 (ordinary training of the last stage)
  norm           root-mean-square norm of activation + residual, with the sum
  norm8          the same with an 8-bit floating output and its scales, one for
                 a row (group 0) or for each `group` columns of it
  norm_grad      the norm's backward: input and gain gradients
  clip           global gradient norm over many tensors, and the clipped
                 gradients

Widths, token counts and vocabularies are those of synth.CONFIGS and of the
codec's timed cases (d = 256 .. 8192, 1 to 32768 tokens, 1024 to 128256 ids).
"""
from __future__ import annotations

import math

import torch

DEV = "cuda"
own = False
TINY = 2.0 ** -100  # the smallest amax that an 8-bit scale is made from
F8 = torch.float8_e4m3fn
F8_MAX = 448.0


# ---------------------------------------------------------------------------
# cases
# ---------------------------------------------------------------------------
def _logits(kind, dtype, n, vocab, top=0, scale=1.0, padded=0.0, masked=0.0):
    return {"kind": kind, "dtype": dtype, "n": n, "vocab": vocab, "top": top, "scale": scale,
            "padded": padded, "masked": masked}


def _norm(kind, dtype, n, d, residual=True, group=0):
    return {"kind": kind, "dtype": dtype, "n": n, "d": d, "residual": residual, "group": group}


def _clip(dtype, d, ff, layers, vocab, pad, clips=True):
    return {"kind": "clip", "dtype": dtype, "d": d, "ff": ff, "layers": layers, "vocab": vocab,
            "pad": pad, "clips": clips}


def listed():
    return [
        # one decoding step of eight sequences: the chosen tokens' log
        # probabilities with five alternatives each, a tenth of the ids forbidden
        dict(_logits("logprobs", "bf16", 8, 32000, top=5, masked=0.1), name="logprobs-decode"),
        # scoring a batch of texts at a temperature, an odd vocabulary (rows start at
        # odd offsets), eight alternatives each
        dict(_logits("logprobs", "bf16", 4999, 50257, top=8, scale=0.7), name="logprobs-score-50257"),
        # the log probabilities of a long text under the widest vocabulary
        dict(_logits("logprobs", "bf16", 8192, 128256), name="logprobs-128256"),
        # the last stage's loss at the benchmark's 8 x 4096 tokens, in training
        dict(_logits("loss", "bf16", 32768, 32000, padded=0.05), name="loss-32000"),
        # a policy's gradient with an entropy bonus, float32 logits
        dict(_logits("logprobs_grad", "f32", 8192, 32000, padded=0.1), name="logprobs-grad-f32"),
        # one token of one sequence in serving: the norm before an 8-bit product
        dict(_norm("norm8", "bf16", 1, 4096), name="norm8-one-token"),
        # an awkward width and an odd number of tokens, a scale for 128 columns
        dict(_norm("norm8", "bf16", 4999, 1600, group=128), name="norm8-d1600-groups"),
        # a block's norm at the benchmark's workload
        dict(_norm("norm", "bf16", 32768, 4096), name="norm-d4096"),
        # its backward at the widest model
        dict(_norm("norm_grad", "bf16", 16383, 8192), name="norm-grad-d8192"),
        # the smallest program: a float32 model of width 256 with four layers
        dict(_clip("f32", 256, 1024, 4, 1024, True), name="clip-tiny-f32"),
        # a model of odd widths whose gradients lie without gaps in one buffer
        dict(_clip("bf16", 1600, 4267, 6, 50257, False), name="clip-d1600-packed"),
        # four layers of width 4096 with their token table
        dict(_clip("bf16", 4096, 14336, 4, 32000, True), name="clip-d4096"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    most = max(work(c)["bytes"] for c in listed())
    while True:
        case = _draw(rng)
        if work(case)["bytes"] <= most:
            return case


def _draw(rng):
    op = rng.choice(["logits", "logits", "norm", "norm", "clip"])
    dtype = "f32" if rng.random() < 0.3 else "bf16"
    if op == "logits":
        vocab = rng.choice([1024, 32000, 50257, 128256, _log_int(rng, 1000, 128256)])
        kind = rng.choice(["logprobs", "logprobs", "loss", "logprobs_grad"])
        lo = 1 if kind == "logprobs" else 64
        return _logits(kind, dtype, _log_int(rng, lo, min(32768, max(256, (1 << 30) // vocab))), vocab,
                       top=rng.choice([0, 1, 5, 8, 20]) if kind == "logprobs" else 0,
                       scale=rng.choice([1.0, 1.0, 0.7, 1.25]),
                       padded=0.0 if kind == "logprobs" else rng.choice([0.0, 0.05, 0.3]),
                       masked=rng.choice([0.0, 0.0, 0.1, 0.9]))
    if op == "norm":
        d = 256 * _log_int(rng, 1, 32) if rng.random() < 0.6 else _log_int(rng, 200, 8192)
        kind = rng.choice(["norm", "norm8", "norm8", "norm_grad"])
        return _norm(kind, dtype, _log_int(rng, 1, 32768), d, residual=rng.random() < 0.8,
                     group=rng.choice([0, 128]) if kind == "norm8" else 0)
    d = 256 * _log_int(rng, 1, 16) if rng.random() < 0.6 else _log_int(rng, 200, 4096)
    return _clip(dtype, d, rng.choice([4 * d, 8 * d // 3, int(3.5 * d)]), _log_int(rng, 1, 24),
                 rng.choice([1024, 32000, 50257]), rng.random() < 0.6, clips=rng.random() < 0.8)


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------
def _type(case):
    return torch.float32 if case["dtype"] == "f32" else torch.bfloat16


def _gen(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(1000003 * int(seed) + sum(ord(c) for c in case["kind"]) + int(case.get("n", 0)))
    return g


def _randn(g, *shape, dtype, std=1.0):
    """A random matrix, made in pieces of rows so that its float32 form stays small."""
    out = torch.empty(shape, dtype=dtype, device=DEV)
    rows = out if out.dim() > 1 else out[None]
    step = max(1, (1 << 27) // max(1, rows.shape[1]))
    for r in range(0, rows.shape[0], step):
        part = rows[r:r + step]
        part.copy_(torch.randn(part.shape, generator=g, device=DEV) * std)
    return out


def prepare(case, seed):
    return {"logprobs": _logit_state, "logprobs_grad": _logit_state, "loss": _logit_state,
            "norm": _norm_state, "norm8": _norm_state, "norm_grad": _norm_state,
            "clip": _clip_state}[case["kind"]](case, seed)


def _logit_state(case, seed):
    g, n, v = _gen(case, seed), case["n"], case["vocab"]
    # logits spread over a few units about a prior that falls with an id's rank
    prior = -torch.log1p(torch.arange(v, device=DEV, dtype=torch.float32))
    Z = torch.empty(n, v, dtype=_type(case), device=DEV)
    allowed = None
    if case["masked"]:
        allowed = torch.rand(v, generator=g, device=DEV) >= case["masked"]
        allowed[0] = True
    step = max(1, (1 << 27) // v)
    for r in range(0, n, step):
        part = Z[r:r + step]
        x = torch.randn(part.shape, generator=g, device=DEV) * 2.5 + prior
        part.copy_(x if allowed is None else torch.where(allowed, x, -math.inf))
    # the given tokens follow the prior, as text does
    u = torch.rand(n, generator=g, device=DEV)
    tok = (torch.exp(u * math.log(v + 1.0)) - 1.0).to(torch.int32).clamp_(0, v - 1)
    if allowed is not None:
        tok = torch.where(allowed[tok.long()], tok, torch.zeros_like(tok))
    pad = torch.rand(n, generator=g, device=DEV) < case["padded"]
    s = {"case": case, "Z": Z, "tok": torch.where(pad, torch.full_like(tok, -1), tok)}
    if case["kind"] == "loss":
        s["weight"] = torch.rand(n, generator=g, device=DEV) * (2.0 / n)
        s["dZ"] = torch.empty_like(Z)
    if case["kind"] == "logprobs_grad":
        # what the forward pass left: each row's largest logit, the logarithm of
        # its sum, and its entropy
        s["stats"], s["entropy"] = torch.empty(n, 2, device=DEV), torch.empty(n, device=DEV)
        for r in range(0, n, step):
            m, logsum, h, _ = _softmax(Z[r:r + step].float(), case["scale"])
            s["stats"][r:r + step] = torch.cat([m, logsum], 1)
            s["entropy"][r:r + step] = h[:, 0]
        s["g_logp"] = torch.randn(n, generator=g, device=DEV) / n
        s["g_entropy"] = torch.full((n,), 0.01 / n, device=DEV)
        s["dZ"] = torch.empty_like(Z)
    return s


def _norm_state(case, seed):
    g, n, d, t = _gen(case, seed), case["n"], case["d"], _type(case)
    w = (1.0 + 0.1 * torch.randn(d, generator=g, device=DEV)).to(t)
    s = {"case": case, "w": w, "X": _randn(g, n, d, dtype=t), "R": None}
    if case["residual"]:
        s["R"] = _randn(g, n, d, dtype=t, std=2.0)
    if case["kind"] == "norm_grad":
        s["dY"] = _randn(g, n, d, dtype=t, std=0.01)
        s["gw"] = torch.zeros(d, device=DEV)
    return s


def _sizes(case):
    """The model's parameters: (rows, columns), or (0, length) for a gain."""
    d, ff = case["d"], case["ff"]
    layer = [(0, d), (d, d), (d, d), (d, d), (d, d), (0, d), (ff, d), (ff, d), (d, ff)]
    return [(case["vocab"], d)] + layer * case["layers"] + [(0, d)]


def _views(flat, sizes, pad):
    """The parameters' places in one buffer, with gaps up to multiples of 128
    values where `pad`; the buffer's length if it is None."""
    views, at = [], 0
    for r, c in sizes:
        n = max(1, r) * c
        if flat is not None:
            views.append(flat[at:at + n].view((r, c) if r else (c,)))
        at += -(-n // 128) * 128 if pad else n
    return at if flat is None else views


def _clip_state(case, seed):
    g, sizes = _gen(case, seed), _sizes(case)
    flat = _randn(g, 1, _views(None, sizes, case["pad"]), dtype=_type(case), std=1e-3)[0]
    n = sum(max(1, r) * c for r, c in sizes)
    out = torch.zeros_like(flat)
    return {"case": case, "grads": _views(flat, sizes, case["pad"]), "flat": out,
            "out": _views(out, sizes, case["pad"]),
            "max_norm": (0.37 if case["clips"] else 2.0) * 1e-3 * math.sqrt(n)}


# ---------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------
def run(s):
    return (_run_own if own else _run_plain)(s["case"]["kind"], s["case"], s)


def _run_own(kind, case, s):
    import paper_2506_01260_amd as sn
    if kind == "logprobs":
        r = sn.sn_token_logprobs(s["Z"], s["tok"], n_top=case["top"], scale=case["scale"])
        return {"logp": r.logp, "entropy": r.entropy, "stats": r.stats, "top_logp": r.top_logp,
                "top_id": r.top_id}
    if kind == "logprobs_grad":
        return {"dZ": sn.sn_token_logprobs_backward(
            s["Z"], s["stats"], s["entropy"], s["tok"], g_logp=s["g_logp"],
            g_entropy=s["g_entropy"], scale=case["scale"], out=s["dZ"])}
    if kind == "loss":
        logp, dZ = sn.sn_token_loss(s["Z"], s["tok"], weight=s["weight"], scale=case["scale"],
                                    out=s["dZ"])
        return {"logp": logp, "dZ": dZ}
    if kind == "norm":
        Y, H = sn.sn_rmsnorm(s["X"], s["w"], residual=s["R"])
        return {"Y": Y, "H": H}
    if kind == "norm8":
        Q, S, H = sn.sn_rmsnorm_quant(s["X"], s["w"], residual=s["R"], group=case["group"])
        return {"Q": Q, "S": S, "H": H}
    if kind == "norm_grad":
        dX = sn.sn_rmsnorm_backward(s["X"], s["dY"], s["w"], dH=s["R"], gw=s["gw"])
        return {"dX": dX, "gw": s["gw"]}
    total = sn.sn_grad_sumsq(s["grads"])
    norm = sn.sn_grad_clip(s["grads"], total, s["max_norm"], out=s["out"])
    return {"norm": norm, "grads": s["flat"]}


def _softmax(z, scale):
    """(largest, log of the sum, entropy, scaled differences) of rows of logits."""
    m = z.amax(1, keepdim=True)
    x = torch.where(m == -math.inf, torch.full_like(z, -math.inf), (z - m) * scale)
    e = torch.exp(x)
    total = e.sum(1, keepdim=True)
    logsum = torch.log(total)
    mean = torch.where(e > 0, e * x, torch.zeros_like(e)).sum(1, keepdim=True) / total
    h = torch.where(total > 0, logsum - mean, torch.zeros_like(total))
    return m, logsum, h, x


def _logp(x, logsum):
    """x - logsum; a row with nothing allowed has probability 0 everywhere."""
    return torch.where(x == -math.inf, x, x - logsum)


def _order(z):
    """Whole numbers in the order of the values, the lowest index first among equals."""
    b = (z + 0.0).view(torch.int32).long()
    b = torch.where(b < 0, -(b & 0x7FFFFFFF), b)
    return b * (1 << 31) + (z.shape[1] - 1 - torch.arange(z.shape[1], device=z.device))


def _at(tok):
    return tok.long().clamp(min=0)[:, None]


def _run_plain(kind, case, s):
    if kind in ("logprobs", "logprobs_grad", "loss"):
        return _plain_logits(kind, case, s["Z"].float(), s)
    if kind == "clip":
        return _plain_clip(s)
    return _plain_norm(kind, case, s)


def _plain_logits(kind, case, z, s):
    scale, tok, given = case["scale"], s["tok"], (s["tok"] >= 0)[:, None]
    if kind == "logprobs_grad":
        m, logsum = s["stats"][:, :1], s["stats"][:, 1:]
        lp = _logp((z - m) * scale, logsum)
        p = torch.exp(lp)
        gl = torch.where(given, s["g_logp"][:, None], torch.zeros_like(m))
        gh = s["g_entropy"][:, None]
        d = torch.where(p > 0, p * (gl + gh * (lp + s["entropy"][:, None])), torch.zeros_like(p))
        d = (-d).scatter_add_(1, _at(tok), gl) * scale
        return {"dZ": d.to(s["Z"].dtype)}
    m, logsum, h, x = _softmax(z, scale)
    logp = torch.where(given, _logp(x.gather(1, _at(tok)), logsum), torch.zeros_like(m))[:, 0]
    if kind == "loss":
        w = torch.where(given, s["weight"][:, None], torch.zeros_like(m))
        d = (w * torch.exp(_logp(x, logsum))).scatter_add_(1, _at(tok), -w) * scale
        return {"logp": logp, "dZ": d.to(s["Z"].dtype)}
    top_logp = top_id = None
    if case["top"]:
        key = torch.topk(_order(z), case["top"], 1).indices
        top_logp, top_id = _logp(x.gather(1, key), logsum), key.int()
    return {"logp": logp, "entropy": h[:, 0], "stats": torch.cat([m, logsum], 1),
            "top_logp": top_logp, "top_id": top_id}


def _plain_norm(kind, case, s, eps=1e-6):
    t, w = s["X"].dtype, s["w"].float()
    h = s["X"].float()
    if kind == "norm_grad":
        dy = s["dY"].float()
        r = torch.rsqrt(h.square().mean(1, keepdim=True) + eps)
        u = dy * w
        dx = r * u - h * (r * r * r * (u * h).mean(1, keepdim=True))
        if s["R"] is not None:
            dx = dx + s["R"].float()
        s["gw"] += (dy * h * r).sum(0)
        return {"dX": dx.to(t), "gw": s["gw"]}
    if s["R"] is not None:
        h = h + s["R"].float()
    y = h * torch.rsqrt(h.square().mean(1, keepdim=True) + eps) * w
    H = h.to(t) if s["R"] is not None else s["X"]
    if kind == "norm":
        return {"Y": y.to(t), "H": H}
    n, d = y.shape
    group = case["group"] or d
    blocks = torch.nn.functional.pad(y, (0, -d % group)).view(n, -1, group)
    S = blocks.abs().amax(2).clamp(min=TINY) / F8_MAX
    Q = (blocks / S[:, :, None]).clamp(-F8_MAX, F8_MAX).view(n, -1)[:, :d].to(F8)
    return {"Q": Q, "S": S, "H": H}


def _plain_clip(s):
    # the squares' sums of one tensor in 32 bits, the tensors' sums in 64
    total = torch.stack([g.float().square().sum() for g in s["grads"]]).double().sum()[None]
    norm = torch.sqrt(total)
    coef = (s["max_norm"] / norm).clamp(max=1.0).float()
    [o.copy_(g.float() * coef) for g, o in zip(s["grads"], s["out"])]
    return {"norm": norm.float(), "grads": s["flat"]}


# ---------------------------------------------------------------------------
# what a pass cannot do without
# ---------------------------------------------------------------------------
def work(case):
    es = 4 if case["dtype"] == "f32" else 2
    if case["kind"] in ("logprobs", "logprobs_grad", "loss"):
        n, v, passes = case["n"], case["vocab"], 1 if case["kind"] == "logprobs" else 2
        return {"bytes": n * v * es * passes + n * (24 + 8 * case["top"]), "flops": n * v * 6 * passes}
    if case["kind"] == "clip":
        n = sum(max(1, r) * c for r, c in _sizes(case))
        return {"bytes": 2 * n * es, "flops": 3 * n}
    n, d, r = case["n"], case["d"], 1 if case["residual"] else 0
    if case["kind"] == "norm8":
        return {"bytes": n * d * (es * (1 + 2 * r) + 1) + 4 * n * -(-d // (case["group"] or d)) + d * es,
                "flops": 6 * n * d}
    if case["kind"] == "norm":
        return {"bytes": n * d * es * (2 + 2 * r) + d * es, "flops": 5 * n * d}
    return {"bytes": n * d * es * (3 + r) + d * (es + 8), "flops": 11 * n * d}


# ---------------------------------------------------------------------------
# the definitions in 64 bits
# ---------------------------------------------------------------------------
def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] in ("logprobs", "logprobs_grad", "loss"):
        return _exact_logits(case, s)
    if case["kind"] == "clip":
        return _exact_clip(s)
    return _exact_norm(case, s)


def _rows(n, width):
    step = max(1, (1 << 26) // width)
    return [slice(r, min(n, r + step)) for r in range(0, n, step)]


def _exact_logits(case, s):
    """p = exp(scale z) / sum exp(scale z); logp = log p; entropy = -sum p log p."""
    kind, parts = case["kind"], []
    n, v = s["Z"].shape
    for b in _rows(n, v):
        a = s["Z"][b].double() * case["scale"]
        top = a.max(1).values
        lse = top + (a - top[:, None]).exp().sum(1).log()
        lp = a - lse[:, None]
        p = lp.exp()
        plogp = p * lp.clamp(min=-1e30)  # 0 log 0 = 0
        h = -plogp.sum(1)
        tok = s["tok"][b].long()
        hit = torch.zeros(len(tok), v, dtype=torch.bool, device=DEV)
        hit[torch.arange(len(tok), device=DEV), tok.clamp(min=0)] = True
        hit &= (tok >= 0)[:, None]
        logp = torch.where(hit, lp, 0.0).sum(1)
        if kind == "logprobs":
            part = {"logp": logp, "entropy": h,
                    "stats": torch.stack([s["Z"][b].double().max(1).values, lse - top], 1),
                    "top_logp": lp.sort(1, descending=True).values[:, :case["top"]] if case["top"] else None}
        elif kind == "loss":
            w = torch.where(tok >= 0, s["weight"][b].double(), 0.0)[:, None]
            part = {"logp": logp, "dZ": case["scale"] * w * (p - hit.double())}
        else:
            gl = torch.where(tok >= 0, s["g_logp"][b].double(), 0.0)[:, None]
            gh = s["g_entropy"][b].double()[:, None]
            part = {"dZ": case["scale"] * (gl * (hit.double() - p) - gh * (plogp + p * h[:, None]))}
        parts.append(part)
    whole = {k: None if parts[0][k] is None else torch.cat([p[k] for p in parts]) for k in parts[0]}
    if kind == "logprobs":
        whole["top_id"] = None
    return whole


def _exact_norm(case, s, eps=1e-6):
    kind, d, parts = case["kind"], case["d"], []
    w, gw = s["w"].double(), torch.zeros(case["d"], dtype=torch.float64, device=DEV)
    for b in _rows(case["n"], d):
        x = s["X"][b].double()
        res = None if s["R"] is None else s["R"][b].double()
        if kind == "norm_grad":
            rms = (x.pow(2).sum(1, keepdim=True) / d + eps).sqrt()
            unit = x / rms
            du = s["dY"][b].double() * w
            dx = (du - unit * (du * unit).sum(1, keepdim=True) / d) / rms
            gw += (s["dY"][b].double() * unit).sum(0)
            parts.append({"dX": dx if res is None else dx + res})
            continue
        h = x if res is None else x + res
        y = w * h / (h.pow(2).sum(1, keepdim=True) / d + eps).sqrt()
        part = {"Y": y, "H": h}
        if kind == "norm8":
            cuts = list(range(0, d, case["group"] or d)) + [d]
            S = torch.stack([y[:, i:j].abs().max(1).values for i, j in zip(cuts, cuts[1:])], 1)
            S = S.clamp(min=TINY) / F8_MAX
            each = torch.cat([S[:, k:k + 1].expand(-1, j - i) for k, (i, j) in enumerate(zip(cuts, cuts[1:]))], 1)
            part = {"Q": y / each, "S": S, "H": h}  # Q before its rounding to 8 bits
        parts.append(part)
    whole = {k: None if parts[0][k] is None else torch.cat([p[k] for p in parts]) for k in parts[0]}
    if kind == "norm_grad":
        whole["gw"] = gw
    return whole


def _exact_clip(s):
    total = sum(float((g.double() ** 2).sum()) for g in s["grads"])
    norm = math.sqrt(total)
    factor = s["max_norm"] / norm if norm > s["max_norm"] else 1.0
    flat = torch.zeros(s["flat"].shape, dtype=torch.float64, device=DEV)
    for g, o in zip(s["grads"], s["out"]):
        at = (o.data_ptr() - s["flat"].data_ptr()) // o.element_size()
        flat[at:at + g.numel()] = g.double().reshape(-1) * factor
    return {"norm": torch.tensor([norm], dtype=torch.float64), "grads": flat}
