"""Measured cases of the operators of the gated feed-forward block: the block itself, activations kept in 8 bits for its backward pass,
and the linear layer whose products are formed in 8 bits.

`own = False` computes the plain form (elementary torch operations in 32 bits, rounded once at the end); `own = True` makes the calls of
`paper_2609_21594_b200.functional`.  Sizes are those of the framework's matrix sets: the tiny layer (d = 256), the 1B-class stack
(2048 x 5632), the Llama-3-8B set (4096 x 14336), the experts (2048 x 1408), and ragged ones.

8 bits: e4m3 codes and, for each block of 1 x 128 (activations) or 128 x 128 (weights) elements, a byte e that stands for 2^(e - 127), the
least power of two (from 2^-127 on) that brings the block's largest magnitude to at most 448.
"""
import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}
BYTES = {"bf16": 2, "fp32": 4}
MOST_FLOPS = 2.9e12


# ------------------------------------------------------------------------------------------------ cases
def listed():
    return [
        # the tiny layer's rows: what a call costs before any arithmetic counts
        {"name": "feed forward tiny", "op": "ffn", "pass": "forward", "tokens": 128, "dim": 256, "hidden": 1024, "dtype": "bf16",
         "activation": "gelu", "keep": "full"},
        # one token of the Llama-3-8B layer: the weights are read once
        {"name": "feed forward token", "op": "ffn", "pass": "forward", "tokens": 1, "dim": 4096, "hidden": 14336, "dtype": "bf16",
         "activation": "silu", "keep": "none"},
        # a long training row of the Llama-3-8B layer
        {"name": "feed forward llama 8192", "op": "ffn", "pass": "forward", "tokens": 8192, "dim": 4096, "hidden": 14336, "dtype": "bf16",
         "activation": "silu", "keep": "full"},
        # the training step's backward pass there
        {"name": "feed forward backward llama 4096", "op": "ffn", "pass": "backward", "tokens": 4096, "dim": 4096, "hidden": 14336,
         "dtype": "bf16", "activation": "silu", "keep": "full"},
        # a step of the 1B-class layer on a ragged row whose activations are kept in 8 bits
        {"name": "feed forward step 8 bit", "op": "ffn", "pass": "step", "tokens": 3001, "dim": 2048, "hidden": 5632, "dtype": "bf16",
         "activation": "silu", "keep": "8bit"},
        # fp32 on sizes that no vector load divides
        {"name": "feed forward backward odd", "op": "ffn", "pass": "backward", "tokens": 389, "dim": 250, "hidden": 1021, "dtype": "fp32",
         "activation": "silu", "keep": "full"},
        # the hidden activations of a Llama-3-8B row, packed for the backward pass
        {"name": "pack llama", "op": "pack", "rows": 8192, "cols": 14336, "dtype": "bf16", "block": 1},
        # a small matrix of weights
        {"name": "pack weights tiny", "op": "pack", "rows": 256, "cols": 1024, "dtype": "fp32", "block": 128},
        # and read back, on odd sizes
        {"name": "unpack odd", "op": "unpack", "rows": 3001, "cols": 5633, "dtype": "bf16", "block": 1},
        # the gate's product of a Llama-3-8B row
        {"name": "linear 8 bit llama", "op": "linear", "pass": "forward", "tokens": 8192, "dim": 4096, "out": 14336},
        # a handful of sequences decoded together
        {"name": "linear 8 bit tokens", "op": "linear", "pass": "forward", "tokens": 16, "dim": 4096, "out": 4096},
        # the backward pass of a 1B-class layer's gate on a ragged row
        {"name": "linear 8 bit backward", "op": "linear", "pass": "backward", "tokens": 4001, "dim": 2048, "out": 5632},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["ffn", "ffn", "pack", "unpack", "linear", "linear"])
    if op in ("pack", "unpack"):
        cols = rng.choice([_log(rng, 1, 14336), 8 * _log(rng, 2, 1792), rng.choice([1024, 2048, 4096, 5632])])
        rows = max(1, min(_log(rng, 1, 16384), (1 << 26) // cols))
        return {"op": op, "rows": rows, "cols": cols, "dtype": rng.choice(["bf16", "bf16", "fp32"]), "block": rng.choice([1, 1, 128])}
    kind = rng.choice(["forward", "backward"] if op == "linear" else ["forward", "backward", "step"])
    per_token = {"forward": 2, "backward": 4, "step": 6}[kind] * (3 if op == "ffn" else 1)
    dtype = "bf16" if op == "linear" else rng.choice(["bf16", "bf16", "bf16", "fp32"])
    if dtype == "fp32":
        dim, hidden = _log(rng, 16, 1024), _log(rng, 16, 2816)
    else:
        dim = rng.choice([256, 1024, 2048, 4096, 8 * _log(rng, 2, 512), 8 * _log(rng, 2, 512), _log(rng, 16, 1000)])
        hidden = rng.choice([1024, 1408, 4096, 5632, 14336, 8 * _log(rng, 2, 1024), 8 * _log(rng, 2, 1024), _log(rng, 16, 2000)])
    tokens = _log(rng, 1, 1024 if dtype == "fp32" else 8192)
    tokens = max(1, min(tokens, int(MOST_FLOPS / 2 / (per_token * dim * hidden))))
    if op == "linear":
        return {"op": op, "pass": kind, "tokens": tokens, "dim": dim, "out": hidden}
    keep = rng.choice(["full", "8bit"]) if kind != "forward" else rng.choice(["full", "none"])
    return {"op": op, "pass": kind, "tokens": tokens, "dim": dim, "hidden": hidden, "dtype": dtype, "activation": rng.choice(["silu", "gelu"]),
            "keep": keep if dtype == "bf16" or kind == "forward" else "full"}


def _blocks(n):
    return (n + 127) // 128


def work(case):
    if case["op"] in ("pack", "unpack"):
        n, scales = case["rows"] * case["cols"], _blocks(case["cols"]) * (case["rows"] if case["block"] == 1 else _blocks(case["rows"]))
        return {"bytes": n * (1 + BYTES[case["dtype"]]) + scales, "flops": 3 * n}
    t, d = case["tokens"], case["dim"]
    if case["op"] == "linear":
        n = case["out"]
        x8, w8 = t * d + t * _blocks(d), n * d + _blocks(n) * _blocks(d)
        if case["pass"] == "forward":
            return {"bytes": 2 * t * d + w8 + 2 * t * n + x8, "flops": 2 * t * n * d}
        return {"bytes": 2 * t * n + x8 + w8 + 2 * t * d + 2 * n * d, "flops": 4 * t * n * d}
    f, e = case["hidden"], BYTES[case["dtype"]]
    x, w = t * d * e, 3 * d * f * e
    kept = {"none": 0, "full": 2 * t * f * e, "8bit": 2 * t * (f + _blocks(f)) + t * (d + _blocks(d))}[case["keep"]]
    if case["pass"] == "forward":
        return {"bytes": 2 * x + w + kept, "flops": 6 * t * d * f}
    if case["pass"] == "step":
        return {"bytes": 4 * x + 2 * w, "flops": 18 * t * d * f}
    return {"bytes": 2 * x + 2 * w + kept + (x if case["keep"] == "full" else 0), "flops": 12 * t * d * f}


# ------------------------------------------------------------------------------------------------ inputs
def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    return g


def prepare(case, seed):
    g = _generator(seed)
    normal = lambda *shape: torch.randn(shape, generator=g, device="cuda")  # noqa: E731
    s = {"op": case["op"], "pass": case.get("pass"), "keep": case.get("keep"), "activation": case.get("activation")}
    if s["op"] in ("pack", "unpack"):
        # rows of unequal size and a few columns that stand out, as hidden activations have
        x = normal(case["rows"], case["cols"]) * torch.exp(normal(case["rows"], 1) * 0.5) * (1 + 10 * (torch.rand(case["cols"], generator=g, device="cuda") < 0.01))
        s["x"], s["block"] = x.to(DTYPES[case["dtype"]]), case["block"]
        if s["op"] == "unpack":
            s["dtype"] = s["x"].dtype
            s["codes"], s["scales"] = _pack(s.pop("x").float(), s["block"])
        return s
    t, d = case["tokens"], case["dim"]
    if s["op"] == "linear":
        n = case["out"]
        s["x"] = normal(t, d).to(torch.bfloat16)
        s["w"] = _pack(normal(n, d) * d ** -0.5, 128)        # laid out once in 8 bits, as a program keeps them
        if s["pass"] == "backward":
            s["x8"] = _pack(s.pop("x").float(), 1)           # what the forward pass kept
            s["dy"] = (normal(t, n) * 1e-3).to(torch.bfloat16)
        return s
    f, e = case["hidden"], DTYPES[case["dtype"]]
    s["x"] = normal(t, d).to(e)                              # a norm's output
    s["w"] = ((normal(f, d) * d ** -0.5).to(e), (normal(f, d) * d ** -0.5).to(e), (normal(d, f) * f ** -0.5).to(e))
    if s["pass"] != "forward":
        s["dy"] = (normal(t, d) * 1e-3).to(e)
    if s["pass"] == "backward":                              # what the forward pass kept
        kept = [(s["x"].float() @ w.float().T) for w in s["w"][:2]]
        if s["keep"] == "full":
            s["kept"] = tuple(k.to(e) for k in kept)
        else:
            s["kept"] = _pack(s.pop("x").float(), 1) + _pack(kept[0], 1) + _pack(kept[1], 1)
    return s


# ------------------------------------------------------------------------------------------------ plain forms, in 32 bits
def _spread(per_block, shape, block):
    """The blocks' values at all elements."""
    return per_block.repeat_interleave(128, 1)[:, :shape[1]].repeat_interleave(block, 0)[:shape[0]]


def _two_to_the(power):
    """2^power for -126 <= power <= 127, exactly (exp2 may be off in its last place, which turns ties)."""
    return ((power + 127).int() << 23).view(torch.float32)


def _pack(x, block):
    """Codes and scales of fp32 x [rows, cols]."""
    rows, cols = x.shape
    r, c = (rows + block - 1) // block, _blocks(cols)
    padded = torch.nn.functional.pad(x.abs(), (0, c * 128 - cols, 0, r * block - rows))
    top = padded.view(r, block, c, 128).amax((1, 3))
    part, power = torch.frexp(top)                           # part in [1/2, 1); 448 = 7/8 * 2^9
    e = torch.where(top == 0, -127, power - 9 + (part > 0.875).int()).clamp(min=-127)
    return (x * _spread(_two_to_the(-e), x.shape, block)).to(torch.float8_e4m3fn), (e + 127).to(torch.uint8)


def _unpack(codes, scales, block):
    return codes.float() * _spread(_two_to_the(scales.int() - 126) * 0.5, codes.shape, block)


def _activate(g, activation):
    """(act(g), act'(g))"""
    if activation == "silu":
        s = torch.sigmoid(g)
        return g * s, s * (1 + g * (1 - s))
    k = math.sqrt(2 / math.pi)
    t = torch.tanh(k * (g + 0.044715 * g * g * g))
    return 0.5 * g * (1 + t), 0.5 * (1 + t) + 0.5 * g * (1 - t * t) * k * (1 + 3 * 0.044715 * g * g)


def _ffn_backward(dy, x, g, u, w, activation):
    a, slope = _activate(g, activation)
    dh = dy @ w[2]
    dg, du = dh * u * slope, dh * a
    return dg @ w[0] + du @ w[1], dg.T @ x, du.T @ x, dy.T @ (a * u)


def _ffn(s):
    e, w = s["w"][0].dtype, [t.float() for t in s["w"]]
    out = []
    if s["pass"] == "backward":
        if s["keep"] == "full":
            x, g, u = s["x"].float(), s["kept"][0].float(), s["kept"][1].float()
        else:
            x, g, u = (_unpack(s["kept"][2 * i], s["kept"][2 * i + 1], 1) for i in range(3))
    else:
        x = s["x"].float()
        g, u = x @ w[0].T, x @ w[1].T
        out.append(((_activate(g, s["activation"])[0] * u) @ w[2].T).to(e))
        if s["pass"] == "forward":
            return tuple(out + ([g.to(e), u.to(e)] if s["keep"] == "full" else []))
        if s["keep"] == "8bit":
            x, g, u = (_unpack(*_pack(t, 1), 1) for t in (x, g, u))
        else:
            g, u = g.to(e).float(), u.to(e).float()
    return tuple(out + [t.to(e) for t in _ffn_backward(s["dy"].float(), x, g, u, w, s["activation"])])


def _linear(s):
    w = _unpack(*s["w"], 128)
    if s["pass"] == "forward":
        x8 = _pack(s["x"].float(), 1)
        return ((_unpack(*x8, 1) @ w.T).to(torch.bfloat16),) + x8
    dy = s["dy"].float()
    dx = _unpack(*_pack(dy, 1), 1) @ w
    return dx.to(torch.bfloat16), (dy.T @ _unpack(*s["x8"], 1)).to(torch.bfloat16)


def run(s):
    if not own:
        if s["op"] == "pack":
            return _pack(s["x"].float(), s["block"])
        if s["op"] == "unpack":
            return _unpack(s["codes"], s["scales"], s["block"]).to(s["dtype"])
        return _linear(s) if s["op"] == "linear" else _ffn(s)
    from paper_2609_21594_b200 import functional as F

    if s["op"] == "pack":
        return F.quantize(s["x"], s["block"])
    if s["op"] == "unpack":
        return F.dequantize(s["codes"], s["scales"], s["dtype"])
    if s["op"] == "linear":
        if s["pass"] == "forward":
            return F.linear_8bit_forward(s["x"], *s["w"])
        return F.linear_8bit_backward(s["dy"], *s["x8"], *s["w"])
    if s["pass"] == "backward":
        return F.feed_forward_backward(s["dy"], s["x"] if s["keep"] == "full" else None, *s["w"], s["kept"], s["activation"])
    y, kept = F.feed_forward_forward(s["x"], *s["w"], s["activation"], s["keep"])
    if s["pass"] == "forward":
        return (y,) + kept
    return (y,) + F.feed_forward_backward(s["dy"], s["x"] if s["keep"] == "full" else None, *s["w"], kept, s["activation"])


# ------------------------------------------------------------------------------------------------ the definitions, in 64 bits
def _power(n):
    """2^n in 64 bits, exactly."""
    return ((n.long() + 1023) << 52).view(torch.float64)


def _exact_pack(x, block):
    """Each block's least power of two by trial, each code the nearest multiple of its binade's step."""
    rows, cols = x.shape
    top = torch.zeros((-(-rows // block), _blocks(cols)), dtype=torch.float64, device=x.device)
    at = (torch.arange(rows, device=x.device)[:, None] // block) * top.shape[1] + torch.arange(cols, device=x.device)[None] // 128
    top.view(-1).scatter_reduce_(0, at.reshape(-1), x.double().abs().reshape(-1), "amax")
    byte = torch.zeros(top.shape, dtype=torch.int64, device=x.device)
    for bit in (128, 64, 32, 16, 8, 4, 2, 1):                # the least byte that is enough: one more than the largest that is not
        more = byte + bit
        byte = torch.where(top > 448 * _power(more - 1 - 127), more, byte)
    scale = _power(byte - 127).view(-1)[at]
    v = x.double() / scale
    step = _power(torch.frexp(v.abs().clamp(min=2.0 ** -6))[1] - 4)
    return torch.round(v / step) * step, byte.to(torch.uint8), scale


def _restored(x, block):
    codes, _, scale = _exact_pack(x, block)
    return codes * scale


def _given(codes, scales, block):
    r, c = torch.arange(codes.shape[0], device="cuda") // block, torch.arange(codes.shape[1], device="cuda") // 128
    return codes.double() * _power(scales.long() - 127)[r][:, c]


def _exact_activation(g, activation):
    if activation == "silu":
        return g / (1 + torch.exp(-g))
    return g / (1 + torch.exp(-2 * math.sqrt(2 / math.pi) * (g + 0.044715 * g ** 3)))        # (1 + tanh z) / 2 = 1 / (1 + e^-2z)


def _exact_ffn(case, s):
    wg, wu, wd = (t.double() for t in s["w"])
    eight = case["keep"] == "8bit"
    out = []
    if case["pass"] == "backward":
        k = s["kept"]
        x, g, u = (_given(k[2 * i], k[2 * i + 1], 1) for i in range(3)) if eight else (s["x"].double(), k[0].double(), k[1].double())
    else:
        x = s["x"].double()
        g, u = torch.einsum("td,fd->tf", x, wg), torch.einsum("td,fd->tf", x, wu)
        out.append(torch.einsum("tf,df->td", _exact_activation(g, case["activation"]) * u, wd))
        if case["pass"] == "forward":
            return tuple(out + ([g, u] if case["keep"] == "full" else []))
        if eight:
            x, g, u = (_restored(t, 1) for t in (x, g, u))
        else:
            g, u = (t.to(s["x"].dtype).double() for t in (g, u))
    dy = s["dy"].double()
    with torch.enable_grad():                                # the derivative by automatic differentiation of the definition
        leaf = g.detach().requires_grad_()
        a = _exact_activation(leaf, case["activation"])
        slope, = torch.autograd.grad(a.sum(), leaf)
    a = a.detach()
    dh = torch.einsum("td,df->tf", dy, wd)
    du, dg = dh * a, dh * u * slope
    return tuple(out + [torch.einsum("tf,fd->td", dg, wg) + torch.einsum("tf,fd->td", du, wu), torch.einsum("tf,td->fd", dg, x),
                        torch.einsum("tf,td->fd", du, x), torch.einsum("td,tf->df", dy, a * u)])


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "pack":
        return _exact_pack(s["x"], s["block"])[:2]
    if case["op"] == "unpack":
        return _given(s["codes"], s["scales"], s["block"])
    if case["op"] == "ffn":
        return _exact_ffn(case, s)
    w = _given(*s["w"], 128)
    if case["pass"] == "forward":
        codes, scales, scale = _exact_pack(s["x"], 1)
        return torch.einsum("tk,nk->tn", codes * scale, w), codes, scales
    return torch.einsum("tn,nk->tk", _restored(s["dy"], 1), w), torch.einsum("tn,tk->nk", s["dy"].double(), _given(*s["x8"], 1))
