"""The checks of `feed_forward_precision` on emulated results: right ones pass, and each rounding that the documentation rules out is seen."""
import pytest
import torch

import feed_forward_precision as fp
import feed_forward_reference as ref

SIZES = [(17, 72, 40), (60, 136, 200), (300, 256, 512)]


def make(tokens, dim, hidden):
    g = torch.Generator().manual_seed(0)
    r = lambda *s: torch.randn(s, generator=g)  # noqa: E731
    return (r(tokens, dim).bfloat16(), (r(hidden, dim) * dim ** -0.5).bfloat16(), (r(hidden, dim) * dim ** -0.5).bfloat16(),
            (r(dim, hidden) * hidden ** -0.5).bfloat16(), (r(tokens, dim) * 1e-3).bfloat16())


@pytest.mark.parametrize("activation", ["silu", "gelu"])
@pytest.mark.parametrize("tokens,dim,hidden", SIZES)
def test_forward(tokens, dim, hidden, activation):
    x, *w, _ = make(tokens, dim, hidden)
    y, g, u = fp.forward(x, *w, activation)
    f = [t.float() for t in (x, *w)]
    in_fp32 = ((ref.act(f[0] @ f[1].T, activation) * (f[0] @ f[2].T)).bfloat16().float() @ f[3].T).bfloat16()
    assert fp.excess(in_fp32, y) <= fp.LIMIT
    h = fp.bf16(ref.act(fp.bf16(g), activation) * fp.bf16(u))                                     # from g and u as they are kept
    assert fp.excess(fp.bf16(h @ w[2].double().T), y) > fp.LIMIT
    a = fp.bf16(fp.bf16(ref.act(g, activation)) * u)                                              # act(g) rounded before it is multiplied
    assert fp.excess(fp.bf16(a @ w[2].double().T), y) > fp.LIMIT


@pytest.mark.parametrize("activation", ["silu", "gelu"])
@pytest.mark.parametrize("tokens,dim,hidden", SIZES)
def test_backward(tokens, dim, hidden, activation):
    x, wg, wu, wd, dy = make(tokens, dim, hidden)
    _, g, u = fp.forward(x, wg, wu, wd, activation)
    g, u = g.bfloat16(), u.bfloat16()
    want = fp.backward(dy, x, g, u, wg, wu, wd, activation)
    f = [t.float() for t in (dy, x, g, u, wg, wu, wd)]
    a, slope = (t.float() for t in ref.act_and_slope(g.double(), activation))
    dh = f[0] @ f[6]
    dg, du, h = ((v.bfloat16().float()) for v in (dh * f[3] * slope, dh * a, a * f[3]))
    right = [v.bfloat16() for v in (dg @ f[4] + du @ f[5], dg.T @ f[1], du.T @ f[1], f[0].T @ h)]
    assert all(fp.excess(a, b) <= fp.LIMIT for a, b in zip(right, want))
    # dh rounded
    d = fp.bf16(dy.double() @ wd.double())
    ad, sd = ref.act_and_slope(g.double(), activation)
    bg, bu = fp.bf16(d * u.double() * sd), fp.bf16(d * ad)
    for got, value in ((bg @ wg.double() + bu @ wu.double(), want[0]), (bg.T @ x.double(), want[1]), (bu.T @ x.double(), want[2])):
        assert fp.excess(fp.bf16(got), value) > fp.LIMIT
    # the two products of dx rounded before they are added
    p, q = dg.double() @ wg.double(), du.double() @ wu.double()
    assert fp.excess(fp.bf16(fp.bf16(p) + fp.bf16(q)), want[0]) > fp.LIMIT


@pytest.mark.parametrize("tokens,dim,hidden", [(40, 72, 264), (60, 136, 200)])
def test_codes(tokens, dim, hidden):
    x, wg, *_ = make(tokens, dim, hidden)
    value, off = ref.product(x.double(), wg.double())
    codes, e = ref.pack((x.float() @ wg.float().T).double(), 1)
    bad, unsure = fp.codes_at_odds(codes, e, value, off)
    assert bad == 0 and unsure < 0.05
    codes, e = ref.pack(fp.bf16(value), 1)                                                        # packed from values rounded to bf16
    assert fp.codes_at_odds(codes, e, value, off)[0] > 20
