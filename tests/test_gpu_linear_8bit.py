"""The 8-bit linear layer against its definition in 64 bits, on the same codes."""
import pytest
import torch

import feed_forward_reference as ref

pytestmark = pytest.mark.gpu

SIZES = [(1, 1, 1), (1, 128, 128), (3, 5, 7), (16, 512, 512), (17, 72, 40), (128, 256, 384), (129, 264, 520), (255, 1000, 130), (256, 640, 1408),
         (700, 1024, 2816), (1300, 520, 264), (2, 4096, 1024), (40, 130, 4096), (300, 16, 32)]


def make(tokens, dim, out, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    r = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
    x = r(tokens, dim) * torch.exp2(torch.randint(-6, 7, (tokens, 1), generator=g, device="cuda").float())
    w = r(out, dim) * torch.exp2(torch.randint(-5, 6, (out, 1), generator=g, device="cuda").float()) * dim ** -0.5
    return x.bfloat16(), w.bfloat16(), (r(tokens, out) * 1e-3).bfloat16()


@pytest.mark.parametrize("tokens,dim,out", SIZES)
def test_forward_and_backward(tokens, dim, out):
    from paper_2609_21594_b200 import functional as F

    x, w, dy = make(tokens, dim, out)
    w8 = F.quantize(w, 128)
    y, *x8 = F.linear_8bit_forward(x, *w8)
    codes, e = ref.pack(x, 1)
    assert torch.equal(x8[0].double(), codes) and torch.equal(x8[1].long(), e)
    xv, wv = ref.unpack(codes, e, 1), ref.unpack(w8[0].float(), w8[1], 128)
    v, off = ref.product(xv, wv)
    assert y.dtype == torch.bfloat16 and ref.worst(y, (v, ref.rounded(v, off, torch.bfloat16))) <= 1
    dx, dw = F.linear_8bit_backward(dy, *x8, *w8)
    v, off = ref.product(ref.unpack(*ref.pack(dy, 1), 1), wv.T)
    assert ref.worst(dx, (v, ref.rounded(v, off, torch.bfloat16))) <= 1
    v, off = ref.product(dy.double().T, xv.T)
    assert ref.worst(dw, (v, ref.rounded(v, off, torch.bfloat16))) <= 1
    alone = F.linear_8bit_backward(dy, *x8, *w8, need=[True, False])
    assert alone[1] is None and torch.equal(alone[0], dx)
    alone = F.linear_8bit_backward(dy, *x8, *w8, need=[False, True])
    assert alone[0] is None and torch.equal(alone[1], dw)


@pytest.mark.parametrize("tokens,dim,out", [(700, 250, 264), (260, 512, 1021), (1100, 301, 643), (1, 5001, 6999), (70, 1000, 1413), (300, 424, 1000)])
def test_odd_rows_on_the_tensor_cores(tokens, dim, out):
    """Products large enough that rows that TMA cannot address are copied for them; codes as `quantize` gives them, and packed together."""
    from paper_2609_21594_b200 import functional as F

    assert tokens * dim * out >= 2 ** 21
    x, w, dy = make(tokens, dim, out)
    w8 = F.quantize(w, 128)
    want = None
    for codes in (w8, tuple(t.contiguous() for t in w8)):
        y, *x8 = F.linear_8bit_forward(x, *codes)
        xv, wv = ref.unpack(x8[0].float(), x8[1], 1), ref.unpack(w8[0].float(), w8[1], 128)
        v, off = ref.product(xv, wv)
        assert y.is_contiguous() and ref.worst(y, (v, ref.rounded(v, off, torch.bfloat16))) <= 1
        for given in (x8, [t.contiguous() for t in x8]):
            dx, dw = F.linear_8bit_backward(dy, *given, *codes)
            v, off = ref.product(ref.unpack(*ref.pack(dy, 1), 1), wv.T)
            assert ref.worst(dx, (v, ref.rounded(v, off, torch.bfloat16))) <= 1
            v, off = ref.product(dy.double().T, xv.T)
            assert ref.worst(dw, (v, ref.rounded(v, off, torch.bfloat16))) <= 1
            if want is None:
                want = (y, dx, dw)
            assert all(torch.equal(a, b) for a, b in zip((y, dx, dw), want))


def test_views_and_shapes():
    """Codes inside wider rows, and at addresses that no wide load takes; x of more than two dimensions."""
    from paper_2609_21594_b200 import functional as F

    x, w, dy = make(24, 256, 384)
    w8 = F.quantize(w, 128)
    y, *x8 = F.linear_8bit_forward(x, *w8)
    grads = F.linear_8bit_backward(dy, *x8, *w8)
    y3, c3, s3 = F.linear_8bit_forward(x.view(2, 3, 4, 256), *w8)
    assert y3.shape == (2, 3, 4, 384) and torch.equal(y3.view(24, 384), y) and c3.shape == (2, 3, 4, 256) and s3.shape == (2, 3, 4, 2)
    for a, b in zip(F.linear_8bit_backward(dy.view(2, 3, 4, 384), c3, s3, *w8), grads):
        assert torch.equal(a.reshape(b.shape), b)
    for left, same in ((16, True), (1, False)):
        big = torch.full((384, 400), 0x7f, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn)      # NaN all around
        big.view(torch.uint8)[:, left:left + 256] = w8[0].view(torch.uint8)
        inside = big[:, left:left + 256]
        y2, *_ = F.linear_8bit_forward(x, inside, w8[1])
        dx2, _ = F.linear_8bit_backward(dy, *x8, inside, w8[1])
        v, off = ref.product(ref.unpack(x8[0].float(), x8[1], 1), ref.unpack(w8[0].float(), w8[1], 128))
        assert ref.worst(y2, (v, ref.rounded(v, off, torch.bfloat16))) <= 1
        if same:
            assert torch.equal(y2, y) and torch.equal(dx2, grads[0])
        v, off = ref.product(ref.unpack(*ref.pack(dy, 1), 1), ref.unpack(w8[0].float(), w8[1], 128).T)
        assert ref.worst(dx2, (v, ref.rounded(v, off, torch.bfloat16))) <= 1


def test_a_token_that_is_not_finite_stays_its_own():
    from paper_2609_21594_b200 import functional as F

    x, w, _ = make(300, 512, 256)
    w8 = F.quantize(w, 128)
    clean, *_ = F.linear_8bit_forward(x, *w8)
    bad = x.clone()
    bad[17, 3], bad[250, 9] = float("nan"), float("-inf")
    y, *_ = F.linear_8bit_forward(bad, *w8)
    rest = torch.ones(300, dtype=torch.bool, device="cuda")
    rest[[17, 250]] = False
    assert torch.isnan(y[17]).all() and torch.isnan(y[250]).all() and torch.equal(y[rest], clean[rest])


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_autograd(dtype):
    from paper_2609_21594_b200 import functional as F

    x, w, dy = make(100, 256, 384)
    w = w.to(dtype)
    lx, lw = x.clone().requires_grad_(), w.clone().requires_grad_()
    y = F.linear_8bit(lx, lw)
    y.backward(dy)
    w8 = F.quantize(w, 128)
    want, *x8 = F.linear_8bit_forward(x, *w8)
    dx, dw = F.linear_8bit_backward(dy, *x8, *w8)
    assert torch.equal(y, want) and torch.equal(lx.grad, dx) and lw.grad.dtype == dtype and torch.equal(lw.grad, dw.to(dtype))
    empty = torch.zeros((0, 256), dtype=torch.bfloat16, device="cuda")
    lw.grad = None
    F.linear_8bit(empty, lw).sum().backward()
    assert lw.grad.shape == w.shape and not lw.grad.any()


def test_refusals():
    from paper_2609_21594_b200 import functional as F

    x, w, dy = make(4, 256, 384)
    w8, x8 = F.quantize(w, 128), F.quantize(x)
    for call in (lambda: F.linear_8bit_forward(x.float(), *w8), lambda: F.linear_8bit_forward(x[:, :128], *w8), lambda: F.linear_8bit_forward(x, *F.quantize(w)),
                 lambda: F.linear_8bit_forward(x, w, w8[1]), lambda: F.linear_8bit_forward(x, w8[0], w8[1].int()), lambda: F.linear_8bit_forward(x.cpu(), *w8),
                 lambda: F.linear_8bit_forward(x, w8[0][:0], w8[1][:0]), lambda: F.linear_8bit_backward(dy[:3], *x8, *w8),
                 lambda: F.linear_8bit_backward(dy.float(), *x8, *w8), lambda: F.linear_8bit_backward(dy[:, :100], *x8, *w8),
                 lambda: F.linear_8bit_backward(dy, *x8, *w8, need=[True]), lambda: F.linear_8bit_backward(dy, x, x8[1], *w8)):
        with pytest.raises(ValueError):
            call()
