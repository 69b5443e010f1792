"""The gate's activation and its slope at every gate that bf16 can hold up to 10^4, against 64 bits, under the bound that the kernels state."""
import math

import pytest
import torch

import feed_forward_reference as ref

pytestmark = pytest.mark.gpu

FAR = 89 * 2.0 ** -126                                       # what the logistic function loses where it is below the least normal number


def gates(some):
    every = torch.arange(1 << 16, device="cuda", dtype=torch.int32).to(torch.int16).view(torch.bfloat16)
    g = every[torch.isfinite(every) & (every.abs() <= 1e4)]
    return g[:: len(g) // 500] if some else g


@pytest.mark.parametrize("some", [False, True])              # CTA pairs, few tokens; CUDA cores for fp32
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("activation", ["silu", "gelu"])
def test_every_gate(activation, dtype, some):
    from paper_2609_21594_b200 import functional as F

    g = gates(some).to(dtype)
    n = g.numel()
    one = lambda *at: torch.zeros((8, 8), device="cuda").index_put_(at, torch.ones((), device="cuda")).to(dtype)  # noqa: E731
    i = lambda k: torch.tensor([k], device="cuda")  # noqa: E731
    first, second = one(i(0), i(0)), one(i(0), i(1))         # g = x[0], u = x[1] = 1; y[0] = h, dx[0] = dg, dx[1] = du
    x = torch.zeros((n, 8), device="cuda", dtype=dtype)
    x[:, 0], x[:, 1] = g, 1
    y, (gate, up) = F.feed_forward_forward(x, first, second, first, activation)
    assert torch.equal(gate[:, 0], g) and (up[:, 0] == 1).all()
    dy = torch.zeros_like(x)
    dy[:, 0] = 1
    dx = F.feed_forward_backward(dy, x, first, second, first, [gate, up], activation)[0]
    v = g.double()
    k, c = (1.0, 0.0) if activation == "silu" else (2 * math.sqrt(2 / math.pi), 0.044715)
    w, dw = k * v * (1 + c * v * v), k * (1 + 3 * c * v * v)
    # (1 + tanh z) / 2 is the logistic function of 2 z, which keeps its digits where 1 + tanh z of 64 bits is off by 2^-53 of 1: a gate of -8 has 10^-15
    s, rest = torch.sigmoid(w), torch.sigmoid(-w)
    a, slope = v * s, s + v * s * rest * dw
    off = (6 + 4 * w.abs().clamp(max=100)) * 2.0 ** -23
    # the second part of the slope, formed of fp32 values: 1 - s is off by s's error or 2^-24, and the products by a few units
    part = a.abs() * dw * (off * s + 2.0 ** -23 + rest * (off + 2.0 ** -21))
    half = ref.half(dtype)
    for got, value, bound in ((y[:, 0], a, off * a.abs()), (dx[:, 1], a, off * a.abs()), (dx[:, 0], slope, off * s + part + FAR * dw)):
        assert torch.isfinite(got).all()
        bound = bound + half * (value.abs() + bound) + FAR
        assert ((got.double() - value).abs() <= bound).all(), float(((got.double() - value).abs() / bound).max())
