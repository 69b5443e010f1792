"""Measured cases of the operators around the matrices that the Muon step trains: layer norm, rotary positions and attention,
each forward and backward.

`own = False` computes the plain form (elementary torch operations in 32 bits, rounded once at the end); `own = True` makes the calls of
`paper_2609_21594_b200.functional`.  Sizes are those of the framework's matrix sets: the tiny layer (d = 256), the 1B-class
stack (d = 2048, 32 query heads and 8 key heads of 64) and the Llama-3-8B set (d = 4096, 32 and 8 heads of 128), and ragged ones.
"""
import math
import random

import numpy as np
import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}
BYTES = {"bf16": 2, "fp32": 4}


# ------------------------------------------------------------------------------------------------ cases
def listed():
    return [
        # one document of the tiny layer: what a call costs before any arithmetic counts
        {"name": "attention forward tiny", "op": "attention", "backward": False, "batch": 1, "length": 128, "docs": 0, "cut": 0,
         "heads": 4, "kv_heads": 4, "dim": 64, "causal": True, "window": 0, "padded": False},
        # a long training context of the Llama-3-8B layer
        {"name": "attention forward llama 8192", "op": "attention", "backward": False, "batch": 1, "length": 8192, "docs": 0, "cut": 0,
         "heads": 32, "kv_heads": 8, "dim": 128, "causal": True, "window": 0, "padded": False},
        # an encoder's padded batch: odd length, a head size between the usual ones, both directions visible
        {"name": "attention forward padded", "op": "attention", "backward": False, "batch": 5, "length": 1531, "docs": 0, "cut": 3,
         "heads": 6, "kv_heads": 2, "dim": 96, "causal": False, "window": 0, "padded": True},
        # the training step's backward pass at the Llama-3-8B layer
        {"name": "attention backward llama 4096", "op": "attention", "backward": True, "batch": 1, "length": 4096, "docs": 0, "cut": 0,
         "heads": 32, "kv_heads": 8, "dim": 128, "causal": True, "window": 0, "padded": False},
        # documents of uneven lengths packed into one row, 1B-class heads
        {"name": "attention backward packed", "op": "attention", "backward": True, "batch": 1, "length": 6000, "docs": 9, "cut": 7,
         "heads": 32, "kv_heads": 8, "dim": 64, "causal": True, "window": 0, "padded": False},
        # a Llama-3-8B layer's norm over one training row, parameters kept in fp32
        {"name": "norm forward llama", "op": "norm", "backward": False, "rows": 8192, "cols": 4096, "dtype": "bf16", "weight": "fp32",
         "center": True},
        {"name": "norm backward llama", "op": "norm", "backward": True, "rows": 8192, "cols": 4096, "dtype": "bf16", "weight": "fp32",
         "center": True},
        # the tiny layer: 128 rows of 256
        {"name": "norm backward tiny", "op": "norm", "backward": True, "rows": 128, "cols": 256, "dtype": "fp32", "weight": "fp32",
         "center": True},
        # without centring, on an odd width that no vector load divides
        {"name": "norm forward odd", "op": "norm", "backward": False, "rows": 3001, "cols": 5633, "dtype": "fp32", "weight": "fp32",
         "center": False},
        # queries and keys of a Llama-3-8B layer over a long context whose frequencies are stretched
        {"name": "rotary forward llama", "op": "rotary", "backward": False, "batch": 1, "length": 8192, "heads": 32, "kv_heads": 8,
         "dim": 128, "rotary": 128, "layout": "half", "dtype": "bf16", "stretch": 8.0, "positions": False},
        # interleaved pairs in half of a 1B-class head, given positions, gradients in fp32
        {"name": "rotary backward ragged", "op": "rotary", "backward": True, "batch": 3, "length": 1021, "heads": 32, "kv_heads": 8,
         "dim": 64, "rotary": 32, "layout": "interleaved", "dtype": "fp32", "stretch": 1.0, "positions": True},
        # a single token of the tiny layer
        {"name": "rotary forward token", "op": "rotary", "backward": False, "batch": 1, "length": 1, "heads": 4, "kv_heads": 4,
         "dim": 64, "rotary": 64, "layout": "half", "dtype": "bf16", "stretch": 1.0, "positions": True},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["attention", "attention", "norm", "rotary"])
    backward = rng.random() < 0.5
    if op == "norm":
        cols = rng.choice([_log(rng, 16, 14336), 8 * _log(rng, 2, 1792), rng.choice([256, 1024, 2048, 4096, 5632])])
        rows = min(_log(rng, 1, 16384), (1 << 25) // cols)
        dtype = rng.choice(["bf16", "fp32"])
        return {"op": op, "backward": backward, "rows": max(1, rows), "cols": cols, "dtype": dtype,
                "weight": rng.choice([dtype, "fp32"]), "center": rng.random() < 0.7}
    dim = rng.choice([64, 64, 128, 128, 96, 80, 72])
    kv = rng.choice([1, 2, 4, 8])
    heads = kv * rng.choice([1, 2, 4])
    if op == "rotary":
        length = _log(rng, 1, 8192)
        return {"op": op, "backward": backward, "batch": rng.randint(1, 4), "length": length, "heads": heads, "kv_heads": kv, "dim": dim,
                "rotary": rng.choice([dim, dim // 2]), "layout": rng.choice(["half", "interleaved"]),
                "dtype": rng.choice(["bf16", "fp32"]), "stretch": rng.choice([1.0, 4.0, 8.0]), "positions": rng.random() < 0.5}
    kind = rng.choice(["plain", "padded", "packed"])
    length = _log(rng, 16, 4096)
    batch = 1 if kind == "packed" else max(1, min(rng.randint(1, 6), 8192 // length))
    causal = kind == "packed" or rng.random() < 0.7
    return {"op": op, "backward": backward, "batch": batch, "length": length,
            "docs": rng.randint(2, 12) if kind == "packed" else 0, "cut": rng.randint(1, 1 << 20) if kind != "plain" else 0,
            "heads": heads, "kv_heads": kv, "dim": dim, "causal": causal,
            "window": rng.choice([0, max(1, length // 3)]) if causal else 0, "padded": kind == "padded"}


def _lengths(case):
    """Tokens of each sequence: the documents of a packed row, the used part of each row of a padded batch, or the whole rows."""
    r = random.Random(case["cut"])
    n, length = case["batch"], case["length"]
    if case["docs"]:
        at = sorted(r.randint(0, length) for _ in range(case["docs"] - 1))
        return [b - a for a, b in zip([0] + at, at + [length])]
    if case["padded"]:
        return [length] + [r.randint(1, length) for _ in range(n - 1)]
    return [length] * n


def _pairs(case):
    """Query-key pairs that the mask leaves, over all sequences."""
    total = 0
    for n in _lengths(case):
        if not case["causal"]:
            total += n * n
        elif not case["window"] or case["window"] >= n:
            total += n * (n + 1) // 2
        else:
            w = case["window"]
            total += w * (w + 1) // 2 + (n - w) * w
    return total


def work(case):
    if case["op"] == "norm":
        n, e, w = case["rows"] * case["cols"], BYTES[case["dtype"]], BYTES[case["weight"]]
        stats = 4 * case["rows"] * (2 if case["center"] else 1)
        params = case["cols"] * w * (2 if case["center"] else 1)
        if case["backward"]:
            return {"bytes": 3 * n * e + stats + case["cols"] * w + params, "flops": 12 * n}
        return {"bytes": 2 * n * e + stats + params, "flops": 8 * n}
    if case["op"] == "rotary":
        tokens = case["batch"] * case["length"]
        n = tokens * (case["heads"] + case["kv_heads"])
        return {"bytes": 2 * n * case["dim"] * BYTES[case["dtype"]] + (4 * tokens if case["positions"] else 0), "flops": 3 * n * case["rotary"]}
    tokens = case["batch"] * case["length"]
    q, kv = tokens * case["heads"] * case["dim"] * 2, tokens * case["kv_heads"] * case["dim"] * 2
    lse = 4 * tokens * case["heads"]
    pairs = _pairs(case) * case["heads"] * case["dim"]
    if case["backward"]:
        return {"bytes": 4 * q + 4 * kv + lse, "flops": 10 * pairs}      # q, o, do, dq; k, v, dk, dv; five products
    return {"bytes": 2 * q + 2 * kv + lse, "flops": 4 * pairs}


# ------------------------------------------------------------------------------------------------ inputs
def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    return g


def _inverse_frequencies(case):
    """base 500000, and for long contexts each frequency stretched by how often it turns within the 8192 positions trained on:
    f below one turn per such context is divided by the stretch, f above four turns is kept, linear in the turns between."""
    half = case["rotary"] // 2
    f = 500000.0 ** (-np.arange(half, dtype=np.float64) / half)
    if case["stretch"] != 1.0:
        keep = np.clip((8192.0 * f / (2 * math.pi) - 1.0) / 3.0, 0.0, 1.0)
        f = f * (keep + (1.0 - keep) / case["stretch"])
    return f


def _norm_inputs(case, seed):
    g, t, w = _generator(seed), DTYPES[case["dtype"]], DTYPES[case["weight"]]
    shape = (case["rows"], case["cols"])
    scale = torch.exp(torch.randn((case["rows"], 1), generator=g, device="cuda") * 0.5)
    x = ((torch.randn(shape, generator=g, device="cuda") + 0.25) * scale).to(t)     # a residual stream: rows of unequal size
    weight = (1 + 0.1 * torch.randn(case["cols"], generator=g, device="cuda")).to(w)
    bias = (0.1 * torch.randn(case["cols"], generator=g, device="cuda")).to(w) if case["center"] else None
    s = {"x": x, "weight": weight, "bias": bias, "eps": 1e-5}
    if case["backward"]:
        s["dy"] = (torch.randn(shape, generator=g, device="cuda") * 1e-3).to(t)
        s["mean"], s["rstd"] = _norm_statistics(x.float(), case["center"], s["eps"])
    return s


def _rotary_inputs(case, seed):
    g, t = _generator(seed), DTYPES[case["dtype"]]
    b, n, h, kv, d = (case[k] for k in ("batch", "length", "heads", "kv_heads", "dim"))
    if case["backward"]:     # gradients, as attention's backward pass leaves them
        q = (torch.randn((b, n, h, d), generator=g, device="cuda") * 1e-3).to(t)
        k = (torch.randn((b, n, kv, d), generator=g, device="cuda") * 1e-3).to(t)
    else:                    # views into a fused projection's output
        fused = torch.randn((b, n, h + 2 * kv, d), generator=g, device="cuda").to(t)
        q, k = fused[:, :, :h], fused[:, :, h:h + kv]
    positions = None
    if case["positions"]:    # documents packed into each row start again at 0; a lone token stands anywhere
        start = torch.randint(0, n, (b, 1), generator=g, device="cuda")
        i = torch.arange(n, device="cuda")[None]
        positions = torch.where(i < start, i, i - start) if n > 1 else torch.randint(0, 100000, (b, 1), generator=g, device="cuda")
        positions = positions.to(torch.int32).contiguous()
    return {"q": q, "k": k, "inv_freq": _inverse_frequencies(case), "layout": case["layout"], "positions": positions}


def _attention_inputs(case, seed):
    g = _generator(seed)
    b, n, h, kv, d = (case[k] for k in ("batch", "length", "heads", "kv_heads", "dim"))
    fused = torch.randn((b, n, h + 2 * kv, d), generator=g, device="cuda").to(torch.bfloat16)      # a fused projection's output
    if case["docs"]:
        fused = fused[0]
    s = {"q": fused[..., :h, :], "k": fused[..., h:h + kv, :], "v": fused[..., h + kv:, :], "causal": case["causal"],
         "window": case["window"], "lens": None, "offsets": None}
    if case["docs"]:
        s["offsets"] = torch.tensor(np.concatenate([[0], np.cumsum(_lengths(case))]), dtype=torch.int32, device="cuda")
    elif case["padded"]:
        s["lens"] = torch.tensor(_lengths(case), dtype=torch.int32, device="cuda")
    if case["backward"]:
        s["do"] = (torch.randn(s["q"].shape, generator=g, device="cuda") * 1e-2).to(torch.bfloat16)
        s["o"], s["lse"] = _attention_forward(s)
    return s


def prepare(case, seed):
    s = {"norm": _norm_inputs, "rotary": _rotary_inputs, "attention": _attention_inputs}[case["op"]](case, seed)
    return dict(s, op=case["op"], backward=case["backward"], center=case.get("center"))


# ------------------------------------------------------------------------------------------------ plain forms, in 32 bits
def _norm_statistics(x, center, eps):
    mean = x.mean(-1) if center else None
    c = x - mean[:, None] if center else x
    return mean, torch.rsqrt(c.square().mean(-1) + eps)


def _norm_forward(s):
    x = s["x"].float()
    mean, rstd = _norm_statistics(x, s["center"], s["eps"])
    y = (x - mean[:, None] if s["center"] else x) * rstd[:, None] * s["weight"].float()
    if s["bias"] is not None:
        y = y + s["bias"].float()
    return (y.to(s["x"].dtype), mean, rstd) if s["center"] else (y.to(s["x"].dtype), rstd)


def _norm_backward(s):
    x, dy = s["x"].float(), s["dy"].float()
    xhat = (x - s["mean"][:, None] if s["center"] else x) * s["rstd"][:, None]
    g = dy * s["weight"].float()
    dx = g - xhat * (g * xhat).mean(-1, keepdim=True)
    if s["center"]:
        dx = dx - g.mean(-1, keepdim=True)
    t, w = s["x"].dtype, s["weight"].dtype
    dx = (dx * s["rstd"][:, None]).to(t)
    dw = (dy * xhat).sum(0).to(w)
    return (dx, dw, dy.sum(0).to(w)) if s["center"] else (dx, dw)


def _rotate(x, cos, sin, layout):
    """x [batch, tokens, heads, dim]; cos, sin [batch, tokens, 1, rotary / 2]; what lies beyond the rotary part is kept."""
    half = cos.shape[-1]
    r = x[..., :2 * half]
    a, b = (r[..., :half], r[..., half:]) if layout == "half" else (r[..., 0::2], r[..., 1::2])
    u, v = a * cos - b * sin, a * sin + b * cos
    turned = torch.cat((u, v), -1) if layout == "half" else torch.stack((u, v), -1).flatten(-2)
    return torch.cat((turned, x[..., 2 * half:]), -1)


def _rotary(s):
    b, n = s["q"].shape[:2]
    p = s["positions"] if s["positions"] is not None else torch.arange(n, device="cuda")[None].expand(b, n)
    # an angle of 100000 radians has no fraction left in 32 bits that could be compared: the product alone is formed in 64
    angle = p.double()[..., None, None] * torch.from_numpy(s["inv_freq"]).cuda()
    angle = torch.remainder(angle, 2 * math.pi).float()
    cos, sin = torch.cos(angle), torch.sin(angle)
    if s["backward"]:
        sin = -sin
    return tuple(_rotate(s[k].float(), cos, sin, s["layout"]).to(s[k].dtype) for k in ("q", "k"))


def _mask(s):
    """[batch or 1, 1, 1, queries, keys]: True where a query may look at a key."""
    n = s["q"].shape[-3]
    i = torch.arange(n, device="cuda")
    m = torch.ones((1, n, n), dtype=torch.bool, device="cuda")
    if s["causal"]:
        m = m & (i[None, :, None] >= i[None, None, :])
    if s["window"]:
        m = m & (i[None, :, None] - i[None, None, :] < s["window"])
    if s["lens"] is not None:
        used = i[None] < s["lens"][:, None]
        m = m & used[:, :, None] & used[:, None, :]
    if s["offsets"] is not None:
        doc = (i[:, None] >= s["offsets"][None, 1:]).sum(-1)
        m = m & (doc[None, :, None] == doc[None, None, :])
    return m[:, None, None]


def _by_kv_head(x, kv):
    """[(batch,) tokens, heads, dim] -> fp32 [batch, kv heads, heads of each, tokens, dim]"""
    x = x.float() if x.dim() == 4 else x.float()[None]
    b, n, h, d = x.shape
    return x.reshape(b, n, kv, h // kv, d).permute(0, 2, 3, 1, 4)


def _by_token(x, like):
    b, kv, g, n, d = x.shape
    return x.permute(0, 3, 1, 2, 4).reshape(like.shape).to(like.dtype)


def _attention_forward(s):
    kv, dim = s["k"].shape[-2:]
    q, k, v = (_by_kv_head(s[x], kv) for x in ("q", "k", "v"))
    a = torch.where(_mask(s), (q @ k.transpose(-1, -2)) * dim ** -0.5, -math.inf)
    top = a.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, 0.0, top)
    a = torch.exp(a - top)
    total = a.sum(-1, keepdim=True)
    o = torch.where(total > 0, (a @ v) / total, 0.0)
    lse = (top + torch.log(total)).squeeze(-1).flatten(1, 2)       # [batch, heads, tokens], -inf where a row sees nothing
    return _by_token(o, s["q"]), lse if s["q"].dim() == 4 else lse[0]


def _attention_backward(s):
    kv, dim = s["k"].shape[-2:]
    q, k, v, o, do = (_by_kv_head(s[x], kv) for x in ("q", "k", "v", "o", "do"))
    lse = s["lse"].reshape(q.shape[:-1])[..., None]
    p = torch.where(_mask(s), torch.exp((q @ k.transpose(-1, -2)) * dim ** -0.5 - lse), 0.0)
    dv = (p.transpose(-1, -2) @ do).sum(2, keepdim=True)
    ds = p * (do @ v.transpose(-1, -2) - (do * o).sum(-1, keepdim=True)) * dim ** -0.5
    return _by_token(ds @ k, s["q"]), _by_token((ds.transpose(-1, -2) @ q).sum(2, keepdim=True), s["k"]), _by_token(dv, s["v"])


def run(s):
    if not own:
        if s["op"] == "norm":
            return _norm_backward(s) if s["backward"] else _norm_forward(s)
        if s["op"] == "rotary":
            return _rotary(s)
        return _attention_backward(s) if s["backward"] else _attention_forward(s)
    from paper_2609_21594_b200 import functional as F

    if s["op"] == "norm":
        if s["backward"]:
            out = F.layer_norm_backward(s["dy"], s["x"], s["weight"], s["mean"], s["rstd"], bias=s["center"])
        else:
            out = F.layer_norm_forward(s["x"], s["weight"], s["bias"], eps=s["eps"], center=s["center"])
        return tuple(t for t in out if t is not None)
    if s["op"] == "rotary":
        return F.rotary_forward((s["q"], s["k"]), s["inv_freq"], layout=s["layout"], positions=s["positions"], inverse=s["backward"])
    mask = {"causal": s["causal"], "window": s["window"], "q_lens": s["lens"], "k_lens": s["lens"], "q_offsets": s["offsets"],
            "k_offsets": s["offsets"]}
    if s["backward"]:
        return F.attention_backward(s["do"], s["q"], s["k"], s["v"], s["o"], s["lse"], **mask)
    return F.attention_forward(s["q"], s["k"], s["v"], **mask)


# ------------------------------------------------------------------------------------------------ the definitions, in 64 bits
def _exact_norm(s):
    x, w = s["x"].double(), s["weight"].double()
    c = x.shape[1]
    if not s["backward"]:
        mu = x.sum(1) / c if s["center"] else torch.zeros_like(x[:, 0])
        rstd = 1 / torch.sqrt(((x - mu[:, None]) ** 2).sum(1) / c + s["eps"])
        y = (x - mu[:, None]) / (1 / rstd)[:, None] * w
        return (y + s["bias"].double(), mu, rstd) if s["center"] else (y, rstd)
    mu = s["mean"].double() if s["center"] else torch.zeros_like(x[:, 0])
    dy, rstd = s["dy"].double(), s["rstd"].double()
    xc = x - mu[:, None]
    gw = torch.einsum("rc,rc,r->c", dy, xc, rstd)
    # the derivative of (x - mu) * rstd, with rstd' = -rstd^3 (x - mu) / c
    along = torch.einsum("rc,rc,c->r", dy, xc, w) / c
    dx = dy * w * rstd[:, None] - xc * (rstd ** 3 * along)[:, None]
    if s["center"]:
        dx -= (torch.einsum("rc,c->r", dy, w) / c * rstd)[:, None]
    return (dx, gw, dy.sum(0)) if s["center"] else (dx, gw)


def _exact_rotary(s):
    out = []
    half = len(s["inv_freq"])
    f = torch.tensor(s["inv_freq"], dtype=torch.float64, device="cuda")
    for x in (s["q"], s["k"]):
        b, n = x.shape[:2]
        pos = torch.arange(n, device="cuda").repeat(b, 1) if s["positions"] is None else s["positions"]
        turn = torch.exp(1j * pos.double()[:, :, None] * f)[:, :, None]
        if s["backward"]:
            turn = turn.conj()
        y = x.double().clone()
        i = torch.arange(half, device="cuda")
        first, second = (i, i + half) if s["layout"] == "half" else (2 * i, 2 * i + 1)
        z = torch.complex(y[..., first], y[..., second]) * turn
        y[..., first], y[..., second] = z.real, z.imag
        out.append(y)
    return tuple(out)


def _exact_attention(case, s):
    packed = s["q"].dim() == 3
    lens = _lengths(case)
    starts = np.concatenate([[0], np.cumsum(lens)])
    h, kv, d = case["heads"], case["kv_heads"], case["dim"]
    zeros = lambda t: torch.zeros(t.shape, dtype=torch.float64, device="cuda")  # noqa: E731
    o, dq, dk, dv = zeros(s["q"]), zeros(s["q"]), zeros(s["k"]), zeros(s["v"])
    lse = torch.full((h, s["q"].shape[0]) if packed else (s["q"].shape[0], h, s["q"].shape[1]), -math.inf, dtype=torch.float64, device="cuda")
    for b, n in enumerate(lens):
        at = (slice(int(starts[b]), int(starts[b]) + n),) if packed else (b, slice(0, n))
        row = torch.arange(n, device="cuda")[:, None]
        hidden = torch.zeros((n, n), dtype=torch.bool, device="cuda")
        if s["causal"]:
            hidden |= row.T > row
        if s["window"]:
            hidden |= row.T <= row - s["window"]
        for j in range(h):
            q, k, v = s["q"][at + (j,)].double(), s["k"][at + (j // (h // kv),)].double(), s["v"][at + (j // (h // kv),)].double()
            a = torch.einsum("qd,kd->qk", q, k).div_(math.sqrt(d)).masked_fill_(hidden, -math.inf)
            where = (j, at[0]) if packed else (b, j, slice(0, n))
            if not s["backward"]:
                e = torch.logsumexp(a, 1)
                lse[where] = e
                o[at + (j,)] = torch.exp(a.sub_(e[:, None])) @ v
                continue
            p = torch.exp(a.sub_(s["lse"][where].double()[:, None]))
            do = s["do"][at + (j,)].double()
            dv[at + (j // (h // kv),)] += p.T @ do
            t = torch.einsum("qd,kd->qk", do, v) - torch.einsum("qd,qd->q", do, s["o"][at + (j,)].double())[:, None]
            t.mul_(p).div_(math.sqrt(d))
            dq[at + (j,)] = t @ k
            dk[at + (j // (h // kv),)] += t.T @ q
    return (dq, dk, dv) if s["backward"] else (o, lse)


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "norm":
        return _exact_norm(s)
    return _exact_rotary(s) if case["op"] == "rotary" else _exact_attention(case, s)
