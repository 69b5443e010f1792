"""Plain 64-bit forms of the feed-forward block, of blocks in 8 bits and of the 8-bit linear layer, each with a bound of what a right kernel may be off
by, element by element.  Shares nothing with the library.

The bounds.  A sum of n products in fp32, in whatever order, is off by at most (n + 2) 2^-23 of the sum of the terms' magnitudes (2^-23 rather
than 2^-24: a tensor core may cut where others round).  A result rounded to its type is off by half a step, eps / 2 of its value.  The
exponential and the quotient of the activation are off by a few units of fp32, or by up to 2^-18 together where the fast units form them."""
import math

import torch

ACT = {torch.bfloat16: 2.0 ** -18, torch.float32: 2.0 ** -20}


def half(dtype):
    return torch.finfo(dtype).eps / 2


def fp32_sum(n):
    return (n + 2) * 2.0 ** -23


def act(g, activation):
    if activation == "silu":
        return g * torch.sigmoid(g)
    return 0.5 * g * (1 + torch.tanh(math.sqrt(2 / math.pi) * (g + 0.044715 * g ** 3)))


def act_and_slope(g, activation):
    with torch.enable_grad():
        leaf = g.detach().clone().requires_grad_()
        a = act(leaf, activation)
        slope, = torch.autograd.grad(a.sum(), leaf)
    return a.detach(), slope


# ------------------------------------------------------------------------------------------------ 8 bits
def scale_bytes(x, block_rows):
    """The least e with max |finite x| <= 448 * 2^(e - 127) in every block, by search."""
    x = x.double()
    x = torch.where(torch.isfinite(x), x.abs(), 0.0)
    rows, cols = x.shape
    r, c = -(-rows // block_rows), -(-cols // 128)
    padded = x.new_zeros((r * block_rows, c * 128))
    padded[:rows, :cols] = x
    top = padded.view(r, block_rows, c, 128).amax((1, 3))
    e = torch.zeros(top.shape, dtype=torch.int64, device=x.device)
    for _ in range(250):
        e += top > 448 * torch.ldexp(torch.ones_like(top), e - 127)
    return e


def spread(per_block, shape, block_rows):
    r = torch.arange(shape[0], device=per_block.device) // block_rows
    return per_block[r][:, torch.arange(shape[1], device=per_block.device) // 128]


def scales_of(e):
    return torch.ldexp(torch.ones(e.shape, dtype=torch.float64, device=e.device), e.long() - 127)


def nearest_e4m3(v):
    """Nearest multiple of the binade's step (2^-9 below 2^-6), ties to even; NaN for what is not finite.  |v| <= 448."""
    exponent = torch.frexp(v.abs().clamp(min=2.0 ** -6))[1] - 1
    step = torch.ldexp(torch.ones_like(v), torch.where(torch.isfinite(v), exponent, 0) - 3)
    return torch.where(torch.isfinite(v), torch.round(v / step) * step, math.nan)


def pack(x, block_rows):
    e = scale_bytes(x, block_rows)
    return nearest_e4m3(x.double() / spread(scales_of(e), x.shape, block_rows)), e


def unpack(codes, e, block_rows):
    return codes.double() * spread(scales_of(e), codes.shape, block_rows)


# ------------------------------------------------------------------------------------------------ products
def product(a, b, ea=0.0, eb=0.0):
    """a b' and its bound, from bounds of a and b."""
    n = a.shape[1]
    off = fp32_sum(n) * (a.abs() @ b.abs().T)
    if torch.is_tensor(ea):
        off = off + ea @ b.abs().T * (1 + fp32_sum(n))
    if torch.is_tensor(eb):
        off = off + a.abs() @ eb.T * (1 + fp32_sum(n))
    return a @ b.T, off


def rounded(v, off, dtype):
    """The bound after rounding to dtype, with the least step of its subnormals."""
    return off + half(dtype) * (v.abs() + off) + torch.finfo(dtype).tiny * torch.finfo(dtype).eps


def feed_forward(x, w_gate, w_up, w_down, activation):
    """{y, gate, up: (value, bound)}; the bounds of gate and up are those of the fp32 sums."""
    t = x.dtype
    x, w_gate, w_up, w_down = (v.double() for v in (x, w_gate, w_up, w_down))
    g, eg = product(x, w_gate)
    u, eu = product(x, w_up)
    a, _ = act_and_slope(g, activation)
    ea = 1.2 * eg + ACT[t] * a.abs()                     # |act'| < 1.2
    h = a * u
    eh = rounded(h, ea * (u.abs() + eu) + a.abs() * eu, t)
    y, ey = product(h, w_down, eh)
    return {"y": (y, rounded(y, ey, t)), "gate": (g, eg), "up": (u, eu)}


def feed_forward_backward(dy, x, g, u, w_gate, w_up, w_down, activation):
    """(dx, dw_gate, dw_up, dw_down), each (value, bound), at the given x, g and u."""
    t = dy.dtype
    dy, x, g, u, w_gate, w_up, w_down = (v.double() for v in (dy, x, g, u, w_gate, w_up, w_down))
    a, slope = act_and_slope(g, activation)
    dh, eh = product(dy, w_down.T)
    dg, du, h = dh * u * slope, dh * a, a * u
    # the slope is a sum of parts no larger than 1.2 + |g|
    edg = rounded(dg, u.abs() * (slope.abs() * eh + (dh.abs() + eh) * ACT[t] * (1.2 + g.abs())), t)
    edu = rounded(du, a.abs() * eh + ACT[t] * (dh.abs() + eh) * a.abs(), t)
    ea = rounded(h, ACT[t] * h.abs(), t)
    p, ep = product(dg, w_gate.T, edg)
    q, eq = product(du, w_up.T, edu)
    dx = p + q
    out = [(dx, ep + eq + 2.0 ** -23 * (p.abs() + q.abs()))]
    out.append(product(dg.T, x.T, edg.T))
    out.append(product(du.T, x.T, edu.T))
    out.append(product(dy.T, h.T, 0.0, ea.T))
    return [(v, rounded(v, e, t)) for v, e in out]


def worst(got, want):
    """Largest |got - value| / bound; at most 1 for a right result.  Both NaN counts as equal."""
    value, off = want
    got = got.double()
    assert got.shape == value.shape and not torch.isnan(off).any()
    return float(((got - value).abs() / off.clamp(min=1e-300)).max()) if got.numel() else 0.0
