"""The gated feed-forward block, forward and backward, against its definition in 64 bits at the sizes where it can go wrong."""
import pytest
import torch

import feed_forward_reference as ref

pytestmark = pytest.mark.gpu

# tokens, dim, hidden: one element, odd sizes, one token, tiles met exactly and missed by one, more tiles than multiprocessors
SIZES = [(1, 1, 1), (3, 5, 7), (1, 256, 1024), (2, 64, 136), (17, 72, 40), (128, 256, 1024), (129, 264, 520), (255, 512, 1408), (256, 128, 256),
         (257, 136, 1000), (700, 1024, 2816), (1300, 520, 264), (5, 2048, 5632), (33, 100, 50)]


def make(tokens, dim, hidden, dtype, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    r = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
    return (r(tokens, dim).to(dtype), (r(hidden, dim) * dim ** -0.5).to(dtype), (r(hidden, dim) * dim ** -0.5).to(dtype),
            (r(dim, hidden) * hidden ** -0.5).to(dtype), (r(tokens, dim) * 1e-3).to(dtype))


@pytest.mark.parametrize("activation", ["silu", "gelu"])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("tokens,dim,hidden", SIZES)
def test_forward(tokens, dim, hidden, dtype, activation):
    from paper_2609_21594_b200 import functional as F

    x, *w, _ = make(tokens, dim, hidden, dtype)
    want = ref.feed_forward(x, *w, activation)
    y, (gate, up) = F.feed_forward_forward(x, *w, activation)
    assert ref.worst(y, want["y"]) <= 1
    for got, name in ((gate, "gate"), (up, "up")):
        assert ref.worst(got, (want[name][0], ref.rounded(*want[name], dtype))) <= 1
    alone, none = F.feed_forward_forward(x, *w, activation, "none")
    assert none == () and ref.worst(alone, want["y"]) <= 1
    packed, kept = F.feed_forward_forward(x, *w, activation, "8bit")
    assert ref.worst(packed, want["y"]) <= 1 and len(kept) == 6
    codes, e = ref.pack(x, 1)
    assert torch.equal(kept[0].double(), codes) and torch.equal(kept[1].long(), e)
    for i, name in ((2, "gate"), (4, "up")):
        value, off = want[name]
        scale = ref.scales_of(kept[i + 1])
        spread = ref.spread(scale, value.shape, 1)
        got = kept[i].double() * spread
        # half a step of e4m3: 2^-4 of the value, or half of 2^-9 scales below 2^-6 scales
        assert ref.worst(got, (value, off + torch.maximum(2.0 ** -4 * (value.abs() + off), 2.0 ** -10 * spread))) <= 1
        # the least scale that is enough, for some values within the bounds
        enough, less = ref.scale_bytes((value.abs() - off).clamp(min=0), 1), ref.scale_bytes(value.abs() + off, 1)
        assert (enough <= kept[i + 1].long()).all() and (kept[i + 1].long() <= less).all()


@pytest.mark.parametrize("keep", ["full", "8bit"])
@pytest.mark.parametrize("activation", ["silu", "gelu"])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("tokens,dim,hidden", SIZES)
def test_backward(tokens, dim, hidden, dtype, activation, keep):
    from paper_2609_21594_b200 import functional as F

    x, *w, dy = make(tokens, dim, hidden, dtype)
    _, kept = F.feed_forward_forward(x, *w, activation, keep)
    if keep == "full":
        at = (x, *kept)
    else:
        at = tuple(ref.unpack(kept[i].float(), kept[i + 1], 1) for i in (0, 2, 4))
    want = ref.feed_forward_backward(dy, *at, *w, activation)
    got = F.feed_forward_backward(dy, x if keep == "full" else None, *w, kept, activation)
    for g, r in zip(got, want):
        assert g.dtype == dtype and ref.worst(g, r) <= 1
    for k in range(4):                                       # each gradient alone: the same bits
        need = [i == k for i in range(4)]
        one = F.feed_forward_backward(dy, x if keep == "full" else None, *w, kept, activation, need)
        assert all((o is None) != n for o, n in zip(one, need)) and torch.equal(one[k], got[k])


def test_against_differences():
    """The block's gradient along random directions, fp32, against differences of the block itself in 64 bits."""
    from paper_2609_21594_b200 import functional as F

    x, *w, dy = make(23, 40, 56, torch.float32)
    for activation in ("silu", "gelu"):
        leaves = [t.clone().requires_grad_() for t in (x, *w)]
        (F.feed_forward(*leaves, activation) * dy).sum().backward()
        g = torch.Generator(device="cuda").manual_seed(5)
        for k, leaf in enumerate(leaves):
            d = torch.randn(leaf.shape, generator=g, device="cuda").double()
            at = [t.double() for t in (x, *w)]
            side = []
            for s in (1e-5, -1e-5):
                moved = list(at)
                moved[k] = moved[k] + s * d
                side.append(float((ref.act(moved[0] @ moved[1].T, activation) * (moved[0] @ moved[2].T) @ moved[3].T * dy.double()).sum()))
            slope = (side[0] - side[1]) / 2e-5
            # fp32 sums of up to 56 terms in three products, and the difference's own error of about 1e-9
            assert abs(float((leaf.grad.double() * d).sum()) - slope) <= 3 * 58 * 2.0 ** -23 * float((leaf.grad.double() * d).abs().sum()) + 1e-8


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_views(dtype):
    """Rows that are part of wider ones, transposed weights, more than two dimensions: the results of contiguous copies."""
    from paper_2609_21594_b200 import functional as F

    x, wg, wu, wd, dy = make(60, 136, 200, dtype)
    y, kept = F.feed_forward_forward(x, wg, wu, wd)
    grads = F.feed_forward_backward(dy, x, wg, wu, wd, kept)

    def inside(t, left, right):
        big = torch.full((t.shape[0], t.shape[1] + left + right), float("nan"), dtype=t.dtype, device="cuda")
        big[:, left:left + t.shape[1]] = t
        return big[:, left:left + t.shape[1]]

    for views in ([inside(t, 8, 16) for t in (x, wg, wu, wd, dy)], [t.T.contiguous().T for t in (x, wg, wu, wd, dy)],
                  [x.view(3, 20, 136), wg, wu, wd, dy.view(3, 20, 136)]):
        vx, vg, vu, vd, vdy = views
        vy, vkept = F.feed_forward_forward(vx, vg, vu, vd)
        assert vy.shape == vx.shape and torch.equal(vy.reshape(60, 136), y) and all(torch.equal(a.reshape(60, 200), b) for a, b in zip(vkept, kept))
        for a, b in zip(F.feed_forward_backward(vdy, vx, vg, vu, vd, vkept), grads):
            assert torch.equal(a.reshape(b.shape), b)
    # one element off the alignment of wide loads: another engine, the same bounds
    views = [inside(t, 1, 2) for t in (x, wg, wu, wd, dy)]
    want = ref.feed_forward(x, wg, wu, wd, "silu")
    vy, vkept = F.feed_forward_forward(*views[:4])
    assert ref.worst(vy, want["y"]) <= 1
    for got, r in zip(F.feed_forward_backward(views[4], views[0], *views[1:4], vkept), ref.feed_forward_backward(dy, x, *vkept, wg, wu, wd, "silu")):
        assert ref.worst(got, r) <= 1


@pytest.mark.parametrize("keep", ["full", "8bit"])
def test_no_tokens(keep):
    from paper_2609_21594_b200 import functional as F

    _, *w, _ = make(1, 64, 128, torch.bfloat16)
    x = torch.zeros((0, 64), dtype=torch.bfloat16, device="cuda", requires_grad=True)
    leaves = [t.requires_grad_() for t in w]
    y = F.feed_forward(x, *leaves, checkpoint=keep)
    assert y.shape == (0, 64)
    y.sum().backward()
    assert all(t.grad.shape == t.shape and not t.grad.any() for t in leaves)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_a_token_that_is_not_finite_stays_its_own(dtype):
    from paper_2609_21594_b200 import functional as F

    x, *w, dy = make(300, 256, 384, dtype)
    clean, _ = F.feed_forward_forward(x, *w)
    bad = x.clone()
    bad[17, 3], bad[250, 9] = float("nan"), float("inf")
    y, kept = F.feed_forward_forward(bad, *w)
    rest = torch.ones(300, dtype=torch.bool, device="cuda")
    rest[[17, 250]] = False
    assert torch.isnan(y[17]).all() and not torch.isfinite(y[250]).all() and torch.equal(y[rest], clean[rest])
    dx = F.feed_forward_backward(dy, bad, *w, kept, need=[True, False, False, False])[0]
    _, kept_clean = F.feed_forward_forward(x, *w)
    assert torch.equal(dx[rest], F.feed_forward_backward(dy, x, *w, kept_clean, need=[True, False, False, False])[0][rest])


@pytest.mark.parametrize("activation", ["silu", "gelu"])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_far_gates(dtype, activation):
    """Gates of all sizes: the activation neither overflows nor turns into NaN, and its slope is 0 or 1 far out."""
    from paper_2609_21594_b200 import functional as F

    big = torch.tensor([0.0, 1e-30, 1.0, -1.0, 30.0, -30.0, 88.0, -88.0, 104.0, -104.0, 1e4, -1e4, 1e12, -1e12], device="cuda").to(dtype)
    n = big.numel()
    x, eye = big[:, None].repeat(1, 8), torch.zeros((8, 8), device="cuda").to(dtype)
    eye[:, 0] = 1
    one = torch.zeros((8, 8), dtype=dtype, device="cuda")
    one[0, 0] = 1
    up = torch.full((n, 8), 0.5, dtype=dtype, device="cuda")
    gate = x.clone()
    dy = torch.ones((n, 8), dtype=dtype, device="cuda")
    dx, dwg, dwu, dwd = F.feed_forward_backward(dy, torch.ones_like(x), one, one, one, [gate, up], activation)
    for got, r in zip((dx, dwg, dwu, dwd), ref.feed_forward_backward(dy, torch.ones_like(x), gate, up, one, one, one, activation)):
        assert torch.isfinite(got).all() and ref.worst(got, r) <= 1


def test_autograd_keeps_what_it_says():
    from paper_2609_21594_b200 import functional as F

    x, *w, dy = make(200, 256, 512, torch.bfloat16)
    for keep in ("full", "8bit"):
        leaves = [t.clone().requires_grad_() for t in (x, *w)]
        y = F.feed_forward(*leaves, checkpoint=keep)
        _, kept = F.feed_forward_forward(x, *w, "silu", keep)
        saved = y.grad_fn.saved_tensors
        assert sum(t is not None and t.dtype == torch.float8_e4m3fn for t in saved) == (3 if keep == "8bit" else 0)
        y.backward(dy)
        for leaf, g in zip(leaves, F.feed_forward_backward(dy, x if keep == "full" else None, *w, kept)):
            assert torch.equal(leaf.grad, g)
        frozen = [t.clone().requires_grad_(i == 2) for i, t in enumerate((x, *w))]
        F.feed_forward(*frozen, checkpoint=keep).backward(dy)
        assert torch.equal(frozen[2].grad, leaves[2].grad) and all(t.grad is None for i, t in enumerate(frozen) if i != 2)
    with torch.no_grad():
        assert F.feed_forward(*leaves).grad_fn is None
    y = F.feed_forward(*leaves)
    with torch.no_grad():
        leaves[1].add_(1)
    with pytest.raises(RuntimeError):
        y.backward(dy)


def test_refusals():
    from paper_2609_21594_b200 import functional as F

    x, wg, wu, wd, dy = make(4, 16, 24, torch.bfloat16)
    _, kept = F.feed_forward_forward(x, wg, wu, wd)
    _, kept8 = F.feed_forward_forward(x, wg, wu, wd, "silu", "8bit")
    for call in (lambda: F.feed_forward_forward(x, wg, wu, wd, "tanh"), lambda: F.feed_forward_forward(x, wg, wu, wd, "silu", "4bit"),
                 lambda: F.feed_forward_forward(x[:, :8], wg, wu, wd), lambda: F.feed_forward_forward(x, wg, wu[:8], wd),
                 lambda: F.feed_forward_forward(x, wg, wu, wd.T), lambda: F.feed_forward_forward(x.half(), wg.half(), wu.half(), wd.half()),
                 lambda: F.feed_forward_forward(x.float(), wg, wu, wd), lambda: F.feed_forward_forward(x, wg[:0], wu[:0], wd[:, :0]),
                 lambda: F.feed_forward_forward(x, wg.cpu(), wu, wd), lambda: F.feed_forward(x, wg, wu, wd, checkpoint="none"),
                 lambda: F.feed_forward_backward(dy, None, wg, wu, wd, kept), lambda: F.feed_forward_backward(dy, x, wg, wu, wd, kept8),
                 lambda: F.feed_forward_backward(dy, x, wg, wu, wd, []), lambda: F.feed_forward_backward(dy, x, wg, wu, wd, [kept[0], kept[1][:3]]),
                 lambda: F.feed_forward_backward(dy, x, wg, wu, wd, [kept[0], kept[1].float()]), lambda: F.feed_forward_backward(dy, x[:3], wg, wu, wd, kept),
                 lambda: F.feed_forward_backward(dy, x, wg, wu, wd, kept, need=[True]),
                 lambda: F.feed_forward_backward(dy, None, wg, wu, wd, kept8[:5] + (kept8[5].int(),)),
                 lambda: F.feed_forward_backward(dy[:2], None, wg, wu, wd, kept8)):
        with pytest.raises(ValueError):
            call()


# products large enough that odd rows are copied for the tensor cores: dim, hidden, both; one token (rows that need no copy but the weights')
ODD = [(700, 250, 264), (260, 256, 1021), (1100, 301, 643), (1, 5001, 6999), (70, 1000, 1413)]


@pytest.mark.parametrize("keep", ["full", "8bit"])
@pytest.mark.parametrize("tokens,dim,hidden", ODD)
def test_odd_rows_on_the_tensor_cores(tokens, dim, hidden, keep):
    from paper_2609_21594_b200 import functional as F

    assert tokens * dim * hidden >= 2 ** 21
    x, *w, dy = make(tokens, dim, hidden, torch.bfloat16)
    want = ref.feed_forward(x, *w, "gelu")
    y, kept = F.feed_forward_forward(x, *w, "gelu", keep)
    assert y.is_contiguous() and ref.worst(y, want["y"]) <= 1
    if keep == "full":
        at = (x, *kept)
        for got, name in zip(kept, ("gate", "up")):
            assert ref.worst(got, (want[name][0], ref.rounded(*want[name], torch.bfloat16))) <= 1
    else:
        at = tuple(ref.unpack(kept[i].float(), kept[i + 1], 1) for i in (0, 2, 4))
    wants = ref.feed_forward_backward(dy, *at, *w, "gelu")
    for contiguous in (False, True):                         # kept as the call gave it, and as a program that copied it has it
        given = tuple(t.contiguous() for t in kept) if contiguous else kept
        got = F.feed_forward_backward(dy, x if keep == "full" else None, *w, given, "gelu")
        for g, r in zip(got, wants):
            assert g.is_contiguous() and ref.worst(g, r) <= 1
    for k in range(4):
        need = [i == k for i in range(4)]
        assert torch.equal(F.feed_forward_backward(dy, x if keep == "full" else None, *w, kept, "gelu", need)[k], got[k])


@pytest.mark.parametrize("tokens,dim,hidden", [(40, 256, 384), (300, 256, 384), (40, 100, 130)])
def test_what_is_kept_in_8_bits_of_values_that_are_not_finite(tokens, dim, hidden):
    """Every engine: a NaN or an infinity in gate or up is kept as NaN and has no share in its block's scale."""
    from paper_2609_21594_b200 import functional as F

    x, wg, wu, wd, _ = make(tokens, dim, hidden, torch.bfloat16)
    _, clean = F.feed_forward_forward(x, wg, wu, wd, "silu", "8bit")
    wg[5] = float("inf")                                     # column 5 of gate: infinities of both signs, or NaN
    wu[7] = float("nan")
    _, kept = F.feed_forward_forward(x, wg, wu, wd, "silu", "8bit")
    for i, bad in ((2, 5), (4, 7)):
        rest = torch.ones(hidden, dtype=torch.bool, device="cuda")
        rest[bad] = False
        assert torch.isnan(kept[i].float()[:, bad]).all() and torch.isfinite(kept[i].float()[:, rest]).all()
        # the scale is that of the other columns: theirs are the codes of the clean product wherever column `bad` was not the largest
        e = ref.scale_bytes(ref.unpack(clean[i].float(), clean[i + 1], 1).masked_fill(~rest, 0.0), 1)
        same = e == clean[i + 1].long()
        spread = ref.spread(same, kept[i].shape, 1) & rest
        assert torch.equal(kept[i + 1][same], clean[i + 1][same]) and torch.equal(kept[i].float()[spread], clean[i].float()[spread])
        assert same.float().mean() > 0.9
