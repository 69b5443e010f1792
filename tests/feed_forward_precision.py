"""What is rounded on the way, and what is not: the documented forms of the feed-forward block in 64 bits with bf16 roundings at the documented places and no
others, and how far a result is from one of them, in units of what its own rounding costs.

A bound for each element has to allow for the worst order of a sum's errors, n 2^-23 of its terms, which from a few hundred terms on is more than a
rounding to bf16.  The norm of all the errors tells them apart.  `excess` is 1 for a result that is the documented value rounded once.  Errors of fp32
sums turn some roundings of what enters the next product: they are a few 2^-24 sqrt(n) of the value, 10^-5 for the thousands of terms here, so that
they turn at most 10^-5 / 2^-8 = 0.3 % of the roundings by 2^-7 to 2^-8: 0.02 of the square of a rounding's own error.  For a product's own sum the
same once more, and a tensor core that cuts instead of rounding adds as much.  One more rounding to bf16 anywhere, which is independent of the others,
adds about 1: a limit of 1.2 lies between."""
import torch

import feed_forward_reference as ref

LIMIT = 1.2


def bf16(v):
    return v.to(torch.bfloat16).double()


def excess(got, value):
    off, alone = got.double() - value, bf16(value) - value
    return float((off * off).sum() / (alone * alone).sum())


def forward(x, w_gate, w_up, w_down, activation):
    """(y, g, u), unrounded at the end; h is rounded once."""
    x, w_gate, w_up, w_down = (t.double() for t in (x, w_gate, w_up, w_down))
    g, u = x @ w_gate.T, x @ w_up.T
    return bf16(ref.act(g, activation) * u) @ w_down.T, g, u


def backward(dy, x, g, u, w_gate, w_up, w_down, activation):
    """(dx, dw_gate, dw_up, dw_down), unrounded at the end; dg, du and h are rounded once, dh is not."""
    dy, x, g, u, w_gate, w_up, w_down = (t.double() for t in (dy, x, g, u, w_gate, w_up, w_down))
    a, slope = ref.act_and_slope(g, activation)
    dh = dy @ w_down
    dg, du, h = bf16(dh * u * slope), bf16(dh * a), bf16(a * u)
    return dg @ w_gate + du @ w_up, dg.T @ x, du.T @ x, dy.T @ h


def codes_at_odds(codes, scales, value, off):
    """Codes and scales of blocks of 1 x 128 that are not those of `value`, where no error within `off` could change them; and the share of the codes that could."""
    enough, less = (ref.scale_bytes(v, 1) for v in ((value.abs() - off).clamp(min=0), value.abs() + off))
    sure = enough == less
    spread = ref.spread(ref.scales_of(enough), value.shape, 1)
    low, high = (ref.nearest_e4m3(((value + s * off) / spread).clamp(-448, 448)) for s in (-1, 1))
    settled = ref.spread(sure, value.shape, 1) & (low == high)
    bad = int((settled & (codes.double() != low)).sum()) + int((sure & (scales.long() != enough)).sum())
    return bad, 1 - float(settled.double().mean())
