"""Layer norm and RMS norm, forward and backward, against the definition in 64 bits.

Tolerances, derived: with u = 2^-24 and sums of at most 16 terms per thread and then a tree (at most 16 + 10 additions), a mean or
mean square is off by at most 32 u times the mean of the absolute terms; y = (x - mean) rstd w + b then by 64 u (|xh w| (1 + k) + |b| +
k |w|), k = mean |x| rstd, and dx likewise with g = dy w.  A result kept in bf16 adds half an ulp, at most 2^-8 of its value.  Gradients of the
parameters add `rows` terms, per block in sequence (at most rows / blocks + 40 additions): n u of the sum of absolute terms."""
import pytest
import torch

import layer_reference as ref

pytestmark = pytest.mark.gpu

COLS = [1, 2, 3, 8, 31, 64, 128, 250, 256, 257, 264, 512, 513, 1000, 1024, 2048, 2050, 4096, 4100, 5633, 8192, 8193, 14336, 16384]


def make(rows, cols, dtype, param, seed=0, ld=None, offset=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    n = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
    ld = cols if ld is None else ld
    base = (n(rows, ld) + 0.5) * torch.exp(n(rows, 1))
    store = torch.full((rows * ld + offset,), float("nan"), dtype=dtype, device="cuda")
    store[offset:] = base.flatten().to(dtype)
    x = store[offset:].view(rows, ld)[:, :cols]
    return x, (1 + 0.2 * n(cols)).to(param), (0.2 * n(cols)).to(param), (n(rows, cols) * 1e-2).to(dtype)


def check_forward(x, w, b, eps, center):
    from paper_2609_21594_b200 import functional as F

    y, mean, rstd = F.layer_norm_forward(x, w, b, eps, center)
    ry, rm, rr = ref.norm(x, w, b, eps, center)
    u = ref.U32
    k = x.double().abs().mean(-1) * rr
    assert ((rstd.double() - rr).abs() <= 64 * u * rr * (1 + k * k)).all()
    if center:
        assert ((mean.double() - rm).abs() <= 32 * u * x.double().abs().mean(-1)).all()
    else:
        assert mean is None
    xh = ref.norm(x, None, None, eps, center)[0]
    wa = 1.0 if w is None else w.double().abs()
    ba = 0.0 if b is None else b.double().abs()
    tol = 64 * u * (xh.abs() * wa * (1 + k * k)[:, None] + ba + k[:, None] * wa) + (ref.U16 * ry.abs() * 1.01 if y.dtype == torch.bfloat16 else 0)
    assert ((y.double() - ry).abs() <= tol).all()
    return mean, rstd


def check_backward(dy, x, w, mean, rstd):
    from paper_2609_21594_b200 import functional as F

    dx, dw, db = F.layer_norm_backward(dy, x, w, mean, rstd)
    xd, dyd = x.double(), dy.double()
    mu = 0.0 if mean is None else mean.double()[:, None]
    r = rstd.double()[:, None]
    xh = (xd - mu) * r
    g = dyd if w is None else dyd * w.double()
    want = r * (g - xh * (g * xh).mean(-1, keepdim=True) - (g.mean(-1, keepdim=True) if mean is not None else 0.0))
    u = ref.U32
    # x - mean cancels: xh is off by u (|x| + |mean|) rstd
    near = u * (xd.abs() + (mu if isinstance(mu, float) else mu.abs())) * r
    tol = 64 * u * r * (g.abs() + xh.abs() * (g * xh).abs().mean(-1, keepdim=True) + g.abs().mean(-1, keepdim=True))
    tol = tol + 4 * r * (near * (g * xh).abs().mean(-1, keepdim=True) + xh.abs() * (g.abs() * near).mean(-1, keepdim=True))
    if dx.dtype == torch.bfloat16:
        tol = tol + ref.U16 * want.abs() * 1.01
    assert ((dx.double() - want).abs() <= tol).all()
    n = min(x.shape[0], 4096) + 64
    for got, terms in ((dw, dyd * xh), (db, dyd)):
        if got is None:
            continue
        s = terms.sum(0)
        t = n * u * terms.abs().sum(0) + 4 * (dyd.abs() * near).sum(0) + (ref.U16 * s.abs() * 1.01 if got.dtype == torch.bfloat16 else 0)
        assert ((got.double() - s).abs() <= t).all()
    return dx, dw, db


@pytest.mark.parametrize("cols", COLS)
@pytest.mark.parametrize("dtype,param", [(torch.bfloat16, torch.float32), (torch.bfloat16, torch.bfloat16), (torch.float32, torch.float32),
                                         (torch.float32, torch.bfloat16)])
@pytest.mark.parametrize("center", [True, False])
def test_every_width(cols, dtype, param, center):
    x, w, b, dy = make(37, cols, dtype, param)
    mean, rstd = check_forward(x, w, b, 1e-5, center)
    check_backward(dy, x, w, mean, rstd)


@pytest.mark.parametrize("rows", [1, 2, 7, 8, 9, 64, 127, 128, 129, 147, 149, 600, 5000])
@pytest.mark.parametrize("cols", [48, 256, 640, 4096, 9000])
def test_row_counts(rows, cols):
    x, w, b, dy = make(rows, cols, torch.bfloat16, torch.float32)
    mean, rstd = check_forward(x, w, b, 1e-5, True)
    check_backward(dy, x, w, mean, rstd)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("cols,ld,offset", [(256, 320, 0), (256, 259, 0), (256, 256, 1), (1000, 1003, 3), (4096, 4104, 8)])
def test_strides_and_alignment(dtype, cols, ld, offset):
    x, w, b, dy = make(19, cols, dtype, torch.float32, ld=ld, offset=offset)
    mean, rstd = check_forward(x, w, b, 1e-5, True)
    check_backward(dy, x, w, mean, rstd)


def test_optional_parameters_and_leading_dimensions():
    from paper_2609_21594_b200 import functional as F

    x, w, b, dy = make(24, 96, torch.float32, torch.float32)
    for weight, bias in ((None, None), (w, None), (None, b)):
        mean, rstd = check_forward(x, weight, bias, 1e-5, True)
        _, dw, db = check_backward(dy, x, weight, mean, rstd)
        assert (dw is None) == (weight is None) and db is not None
    y3, m3, r3 = F.layer_norm_forward(x.view(2, 3, 4, 96), w, b)
    y2, m2, r2 = F.layer_norm_forward(x, w, b)
    assert torch.equal(y3.view(24, 96), y2) and m3.shape == r3.shape == (2, 3, 4) and torch.equal(r3.flatten(), r2)
    y1, _, r1 = F.layer_norm_forward(x[5], w, b)
    assert torch.equal(y1, y2[5]) and r1.shape == ()


def test_no_rows():
    from paper_2609_21594_b200 import functional as F

    x = torch.empty((0, 300), device="cuda")
    w = torch.ones(300, device="cuda")
    y, mean, rstd = F.layer_norm_forward(x, w, w)
    assert y.shape == (0, 300) and rstd.shape == (0,)
    dx, dw, db = F.layer_norm_backward(y, x, w, mean, rstd)
    assert dx.shape == (0, 300) and not dw.any() and not db.any()


def test_large_offset_rows_keep_their_variance():
    """A row of 1000 +- 1e-2: the variance comes from centred values."""
    from paper_2609_21594_b200 import functional as F

    g = torch.Generator(device="cuda").manual_seed(1)
    x = 1000 + 1e-2 * torch.randn((4, 4096), generator=g, device="cuda")
    _, _, rstd = F.layer_norm_forward(x, eps=0.0)
    _, _, want = ref.norm(x, None, None, 0.0, True)
    # the mean is off by at most 32 u 1000 = 1.9e-3; its square adds to a variance of 1e-4
    assert ((rstd.double() / want - 1).abs() <= 0.5 * (32 * ref.U32 * 1000) ** 2 / 1e-4 + 64 * ref.U32 * 1e5).all()


def test_special_values_stay_in_their_row():
    from paper_2609_21594_b200 import functional as F

    x, w, b, dy = make(40, 512, torch.bfloat16, torch.float32)
    clean, _, _ = F.layer_norm_forward(x, w, b)
    x = x.clone()
    x[3, 7], x[20, 0] = float("nan"), float("inf")
    y, mean, rstd = F.layer_norm_forward(x, w, b)
    keep = torch.ones(40, dtype=torch.bool, device="cuda")
    keep[[3, 20]] = False
    assert torch.equal(y[keep], clean[keep]) and y[3].isnan().all() and y[20].isnan().any()
    zero, _, r0 = F.layer_norm_forward(torch.zeros((2, 64), device="cuda"), eps=1e-5)
    assert not zero.any() and torch.allclose(r0, torch.full_like(r0, 1e-5 ** -0.5))


def test_same_bits_every_time_and_on_another_stream():
    from paper_2609_21594_b200 import functional as F

    x, w, b, dy = make(3000, 2048, torch.bfloat16, torch.float32)
    y, mean, rstd = F.layer_norm_forward(x, w, b)
    first = F.layer_norm_backward(dy, x, w, mean, rstd)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        second = F.layer_norm_backward(dy, x, w, mean, rstd)
        y2 = F.layer_norm_forward(x, w, b)[0]
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(y, y2) and all(torch.equal(a, b) for a, b in zip(first, second))


def test_in_place():
    from paper_2609_21594_b200 import binding as mb
    from paper_2609_21594_b200 import functional as F

    x, w, b, dy = make(50, 1024, torch.bfloat16, torch.float32)
    y, mean, rstd = F.layer_norm_forward(x, w, b)
    dx, _, _ = F.layer_norm_backward(dy, x, w, mean, rstd)
    desc = mb.NormDesc(mb.DTYPE_BF16, mb.DTYPE_FP32, 1, 1024, 50, 1e-5, 0)
    c = F.context()
    inplace, grad, over = x.clone(), dy.clone(), x.clone()
    c.muon_layer_norm_forward(desc, inplace.data_ptr(), 1024, w.data_ptr(), b.data_ptr(), inplace.data_ptr(), 1024, mean.data_ptr(), rstd.data_ptr())
    c.muon_layer_norm_backward(desc, grad.data_ptr(), 1024, x.data_ptr(), 1024, w.data_ptr(), mean.data_ptr(), rstd.data_ptr(), grad.data_ptr(), 1024,
                               None, None, None, 0)
    c.muon_layer_norm_backward(desc, dy.data_ptr(), 1024, over.data_ptr(), 1024, w.data_ptr(), mean.data_ptr(), rstd.data_ptr(), over.data_ptr(), 1024,
                               None, None, None, 0)
    assert torch.equal(inplace, y) and torch.equal(grad, dx) and torch.equal(over, dx)


@pytest.mark.parametrize("center", [True, False])
def test_autograd_against_differences(center):
    """fp32: <gradient, direction> against the central difference of the 64-bit loss.  The difference is off by h^2 / 6 times the third
    derivative, about 1e-8 of the loss scale at h = 1e-4 in 64 bits; the gradient by 64 u of the sum of absolute terms: 1e-4 covers both."""
    from paper_2609_21594_b200 import functional as F

    x, w, b, _ = make(6, 200, torch.float32, torch.float32)
    g = torch.Generator(device="cuda").manual_seed(5)
    x, w, b = (t.clone().requires_grad_() for t in (x, w, b))
    c = torch.randn(x.shape, generator=g, device="cuda")
    F.layer_norm(x, w, b, 1e-5, center).backward(c)
    loss = lambda x, w, b: (ref.norm(x, w, b, 1e-5, center)[0] * c.double()).sum()  # noqa: E731
    h = 1e-4
    for i, t in enumerate((x, w, b)):
        d = torch.randn(t.shape, generator=g, device="cuda").double()
        hi, lo = [t.detach().double() for t in (x, w, b)], [t.detach().double() for t in (x, w, b)]
        hi[i] = hi[i] + h * d
        lo[i] = lo[i] - h * d
        diff = float(loss(*hi) - loss(*lo)) / (2 * h)
        got = float((t.grad.double() * d).sum())
        assert abs(got - diff) <= 1e-4 * float((t.grad.double() * d).abs().sum())


def test_refusals():
    from paper_2609_21594_b200 import binding as mb
    from paper_2609_21594_b200 import functional as F

    x = torch.zeros((4, 64), device="cuda")
    w = torch.ones(64, device="cuda")
    y, mean, rstd = F.layer_norm_forward(x, w, w)
    with pytest.raises(ValueError):
        F.layer_norm_forward(x.half(), w, w)
    with pytest.raises(ValueError):
        F.layer_norm_forward(x.cpu(), w, w)
    with pytest.raises(ValueError):
        F.layer_norm_forward(x, w[:63], None)
    with pytest.raises(ValueError):
        F.layer_norm_forward(x, w, w.bfloat16())
    with pytest.raises(ValueError):
        F.layer_norm_forward(x[:, :0])
    with pytest.raises(ValueError):
        F.layer_norm_backward(y[:2], x, w, mean, rstd)
    with pytest.raises(ValueError):
        F.layer_norm_backward(y, x, w, mean.double(), rstd)
    for eps in (-1.0, float("nan"), float("inf")):
        with pytest.raises(mb.MuonError) as e:
            F.layer_norm_forward(x, eps=eps)
        assert e.value.code == mb.ERR_INVALID_ARG
    with pytest.raises(mb.MuonError) as e:
        F.layer_norm_forward(torch.zeros((2, 16385), device="cuda"))
    assert e.value.code == mb.ERR_UNSUPPORTED
    c, p = F.context(), x.data_ptr()
    desc = mb.NormDesc(mb.DTYPE_FP32, mb.DTYPE_FP32, 1, 64, 4, 1e-5, 0)
    bad = [lambda: c.muon_layer_norm_forward(desc, None, 64, None, None, p, 64, p, p),
           lambda: c.muon_layer_norm_forward(desc, p, 63, None, None, p, 64, p, p),
           lambda: c.muon_layer_norm_forward(desc, p, 64, None, None, y.data_ptr(), 64, None, rstd.data_ptr()),
           lambda: c.muon_layer_norm_forward(desc, p + 2, 64, None, None, y.data_ptr(), 64, mean.data_ptr(), rstd.data_ptr()),
           lambda: c.muon_layer_norm_forward(mb.NormDesc(7, 1, 1, 64, 4, 1e-5, 0), p, 64, None, None, p, 64, p, p),
           lambda: c.muon_layer_norm_forward(mb.NormDesc(1, 1, 1, 64, -1, 1e-5, 0), p, 64, None, None, p, 64, p, p),
           lambda: c.muon_layer_norm_forward(mb.NormDesc(1, 1, 1, 64, 4, 1e-5, 3), p, 64, None, None, p, 64, p, p)]
    before = c.muon_launch_count()
    for call in bad:
        with pytest.raises(mb.MuonError) as e:
            call()
        assert e.value.code == mb.ERR_INVALID_ARG
    with pytest.raises(mb.MuonError) as e:
        many = mb.NormDesc(mb.DTYPE_FP32, mb.DTYPE_FP32, 1, 64, 1000, 1e-5, 0)      # enough rows to need scratch
        c.muon_layer_norm_backward(many, p, 64, p, 64, None, mean.data_ptr(), rstd.data_ptr(), y.data_ptr(), 64, w.data_ptr(), None, None, 0)
    assert e.value.code == mb.ERR_WORKSPACE_TOO_SMALL
    assert c.muon_launch_count() == before
