"""Rotary positions against the definition in 64 bits.

Tolerance, derived: the angle's fraction is exact to 2^-25 turns (fp32 rounding of a fraction below one half), so cosine and sine are off
by at most 2 pi 2^-25 + 2^-23 < 2.6e-7 + what sincospif adds (2 ulp, 2.4e-7); the turned pair by 6e-7 (|a| + |b|) with two products
and a sum at 2^-24 each; for angles formed in double at position p the reference and the kernel agree to p 2^-52.  bf16 adds half
an ulp."""
import numpy as np
import pytest
import torch

import layer_reference as ref

pytestmark = pytest.mark.gpu


def freq(pairs, base=10000.0):
    return base ** (-np.arange(pairs) / pairs)


def check(xs, f, layout, pos, inverse=False, amplitude=1.0, out=None, **kw):
    from paper_2609_21594_b200 import functional as F

    before = [x.clone() for x in xs]
    got = F.rotary_forward(xs, f, layout=layout, inverse=inverse, amplitude=amplitude, out=out, **kw)
    for x, y in zip(before, got):
        x4, y4 = (x, y) if x.dim() == 4 else (x[None], y[None])
        want = ref.turn(x4, f, pos, layout, amplitude, inverse)
        n = 2 * len(f)
        size = ref.turn(x4.abs(), f, torch.zeros_like(pos), layout, amplitude, inverse)   # |amplitude x|
        ia = torch.arange(len(f), device="cuda") if layout == "half" else 2 * torch.arange(len(f), device="cuda")
        ib = ia + len(f) if layout == "half" else ia + 1
        both = size.abs().clone()
        both[..., ia] = both[..., ib] = size.abs()[..., ia] + size.abs()[..., ib]
        tol = 1e-6 * both + (ref.U16 * want.abs() * 1.01 if x.dtype == torch.bfloat16 else 0)
        assert ((y4.double() - want).abs() <= tol)[..., :n].all()
        assert torch.equal(y4[..., n:], x4[..., n:])
    return got


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("d,pairs", [(2, 1), (6, 3), (64, 32), (64, 16), (64, 8), (96, 24), (100, 50), (128, 64), (128, 20), (80, 13), (256, 128), (512, 256)])
@pytest.mark.parametrize("inverse", [False, True])
def test_layouts_and_sizes(dtype, layout, d, pairs, inverse):
    g = torch.Generator(device="cuda").manual_seed(d + pairs)
    q, k = (torch.randn((2, 37, h, d), generator=g, device="cuda").to(dtype) for h in (3, 1))
    pos = torch.arange(37, device="cuda")[None].expand(2, 37)
    check([q, k], freq(pairs), layout, pos, inverse)


@pytest.mark.parametrize("b,n,heads", [(1, 1, (1,)), (1, 1, (4, 4)), (3, 1, (32, 8)), (1, 2, (1,)), (5, 301, (6, 2, 2)), (1, 4097, (2, 1)), (2, 64, (1, 2, 3, 4))])
def test_token_and_head_counts(b, n, heads):
    g = torch.Generator(device="cuda").manual_seed(n)
    xs = [torch.randn((b, n, h, 64), generator=g, device="cuda").bfloat16() for h in heads]
    check(xs, freq(32), "half", torch.arange(n, device="cuda")[None].expand(b, n))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_views_strides_and_odd_alignment(dtype, layout):
    g = torch.Generator(device="cuda").manual_seed(2)
    pos = torch.arange(29, device="cuda")[None].expand(2, 29)
    fused = torch.randn((2, 29, 12, 64), generator=g, device="cuda").to(dtype)
    check([fused[:, :, :8], fused[:, :, 8:10]], freq(32), layout, pos)
    by_head = torch.randn((2, 5, 29, 64), generator=g, device="cuda").to(dtype).transpose(1, 2)
    check([by_head], freq(32), layout, pos)
    odd = torch.randn((2 * 29 * 3 * 67 + 1,), generator=g, device="cuda").to(dtype)[1:].view(2, 29, 3, 67)[..., :64]
    check([odd], freq(32), layout, pos)
    check([torch.randn((29, 3, 64), generator=g, device="cuda").to(dtype)], freq(16), layout, pos[:1])


def test_positions_offset_and_amplitude():
    g = torch.Generator(device="cuda").manual_seed(3)
    x = torch.randn((2, 33, 2, 64), generator=g, device="cuda")
    p = torch.randint(-50, 131072, (2, 33), generator=g, device="cuda").to(torch.int32)
    check([x], freq(32), "half", p.long(), positions=p, amplitude=1.25)
    check([x], freq(32), "interleaved", p.long() + 7, positions=p, offset=7)
    check([x], freq(32), "half", 1000 + torch.arange(33, device="cuda")[None].expand(2, 33), offset=1000)


def test_far_positions_keep_their_precision():
    """At two billion a product in fp32 would have no fraction left; in double the angle is good to 2^31 2^-52 = 5e-7."""
    from paper_2609_21594_b200 import functional as F

    g = torch.Generator(device="cuda").manual_seed(4)
    x = torch.randn((1, 8, 1, 64), generator=g, device="cuda")
    p = (2 ** 31 - 1 - torch.arange(8, device="cuda"))[None].to(torch.int32)
    y = F.rotary_forward([x], freq(32), positions=p)[0]
    want = ref.turn(x, freq(32), p.long(), "half", 1.0, False)
    # the table in turns and the product are rounded at 2^-53 each, as are the reference's angles: 3 * 2^31 * 2^-53 radians, and the above
    assert ((y.double() - want).abs() <= (1e-6 + 3 * 2.0 ** -22) * (x.abs().amax() * 2)).all()


@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_in_place_and_back(layout):
    from paper_2609_21594_b200 import functional as F

    g = torch.Generator(device="cuda").manual_seed(6)
    x = torch.randn((2, 50, 4, 96), generator=g, device="cuda")
    y = F.rotary_forward([x], freq(32), layout=layout)[0]
    z = x.clone()
    check([z], freq(32), layout, torch.arange(50, device="cuda")[None].expand(2, 50), out=[z])
    assert torch.equal(z, y)
    back = F.rotary_forward([y], freq(32), layout=layout, inverse=True)[0]
    assert ((back - x).abs() <= 4e-6 * x.abs().amax()).all()


@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_autograd_is_the_transpose(layout):
    """<R x, c> = <x, R^T c>, and the map is linear, so a difference quotient is exact: both sides to 1e-6 of the absolute sum."""
    from paper_2609_21594_b200 import functional as F

    g = torch.Generator(device="cuda").manual_seed(7)
    q, k = (torch.randn((1, 21, h, 64), generator=g, device="cuda", requires_grad=True) for h in (4, 2))
    cq, ck = torch.randn(q.shape, generator=g, device="cuda"), torch.randn(k.shape, generator=g, device="cuda")
    yq, yk = F.rotary([q, k], freq(24), layout)
    torch.autograd.backward([yq, yk], [cq, ck])
    pos = torch.arange(21, device="cuda")[None]
    for x, c in ((q, cq), (k, ck)):
        d = torch.randn(x.shape, generator=g, device="cuda")
        h = 0.5
        diff = ((ref.turn(x.detach() + h * d, freq(24), pos, layout, 1.0, False) - ref.turn(x.detach() - h * d, freq(24), pos, layout, 1.0, False)) * c).sum() / (2 * h)
        assert abs(float((x.grad.double() * d).sum() - diff)) <= 2e-6 * float((x.grad * d).abs().sum()) + 2e-6 * float((c * d).abs().sum())


def test_refusals_and_empty_calls():
    from paper_2609_21594_b200 import binding as mb
    from paper_2609_21594_b200 import functional as F

    x = torch.zeros((1, 4, 2, 64), device="cuda")
    for call in (lambda: F.rotary_forward([], freq(8)), lambda: F.rotary_forward([x] * 5, freq(8)), lambda: F.rotary_forward([x], freq(33)),
                 lambda: F.rotary_forward([x], freq(8), layout="other"), lambda: F.rotary_forward([x, x[:, :3]], freq(8)),
                 lambda: F.rotary_forward([x], freq(8), positions=torch.zeros(4, device="cuda")),
                 lambda: F.rotary_forward([x], freq(8), positions=torch.zeros(3, dtype=torch.int32, device="cuda")),
                 lambda: F.rotary_forward([x.half()], freq(8)), lambda: F.rotary_forward([x.cpu()], freq(8)),
                 lambda: F.rotary_forward([x], freq(8), out=[x[:, :2]])):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(mb.MuonError) as e:
        F.rotary_forward([x], freq(8), amplitude=float("nan"))
    assert e.value.code == mb.ERR_INVALID_ARG
    with pytest.raises(mb.MuonError) as e:
        F.rotary_forward([x], freq(8), out=[x.transpose(0, 1).contiguous().transpose(0, 1)[:, :, :1].expand(1, 4, 2, 64)])
    assert e.value.code == mb.ERR_INVALID_ARG          # two heads of the result share a place
    for shape in ((0, 4, 2, 64), (1, 0, 2, 64), (1, 4, 0, 64)):
        assert F.rotary_forward([torch.zeros(shape, device="cuda")], freq(8))[0].shape == shape
