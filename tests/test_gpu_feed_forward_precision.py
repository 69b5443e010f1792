"""The feed-forward block and the 8-bit linear layer round where the documentation says and nowhere else, on every engine."""
import pytest
import torch

import feed_forward_precision as fp
import feed_forward_reference as ref

pytestmark = pytest.mark.gpu

# few tokens, CTA pairs with narrow and with wide tiles, odd rows by way of copies; and, off the alignment of wide loads, CUDA cores
SIZES = [(17, 72, 40, 0), (5, 2048, 1408, 0), (60, 136, 200, 0), (700, 1024, 2816, 0), (3000, 512, 1408, 0), (260, 256, 1021, 0), (60, 136, 200, 1), (300, 256, 520, 1)]


def make(tokens, dim, hidden, left):
    g = torch.Generator(device="cuda").manual_seed(0)

    def r(rows, cols, scale):
        wide = torch.zeros((rows, cols + 8), dtype=torch.bfloat16, device="cuda") if left else torch.empty((rows, cols), dtype=torch.bfloat16, device="cuda")
        out = wide[:, left:left + cols]
        return out.copy_(torch.randn((rows, cols), generator=g, device="cuda") * scale)

    return r(tokens, dim, 1), r(hidden, dim, dim ** -0.5), r(hidden, dim, dim ** -0.5), r(dim, hidden, hidden ** -0.5), r(tokens, dim, 1e-3)


@pytest.mark.parametrize("activation", ["silu", "gelu"])
@pytest.mark.parametrize("tokens,dim,hidden,left", SIZES)
def test_block(tokens, dim, hidden, left, activation):
    from paper_2609_21594_b200 import functional as F

    x, *w, dy = make(tokens, dim, hidden, left)
    y, g, u = fp.forward(x, *w, activation)
    for keep in ("full", "8bit", "none"):
        got, kept = F.feed_forward_forward(x, *w, activation, keep)
        assert fp.excess(got, y) <= fp.LIMIT, keep
        if keep == "none":
            continue
        at = (x, *kept) if keep == "full" else tuple(ref.unpack(kept[i].float(), kept[i + 1], 1) for i in (0, 2, 4))
        if keep == "full":
            assert fp.excess(kept[0], g) <= fp.LIMIT and fp.excess(kept[1], u) <= fp.LIMIT
        grads = F.feed_forward_backward(dy, x if keep == "full" else None, *w, kept, activation)
        for k, (a, b) in enumerate(zip(grads, fp.backward(dy, *at, *w, activation))):
            assert fp.excess(a, b) <= fp.LIMIT, (keep, k)


@pytest.mark.parametrize("tokens,dim,hidden,left", [(40, 72, 264, 0), (300, 136, 384, 0), (1500, 64, 1000, 0), (40, 100, 130, 0), (300, 136, 384, 1)])
def test_gate_and_up_are_packed_from_the_fp32_sums(tokens, dim, hidden, left):
    from paper_2609_21594_b200 import functional as F

    x, *w, _ = make(tokens, dim, hidden, left)
    _, kept = F.feed_forward_forward(x, *w, "silu", "8bit")
    for i, weight in ((2, w[0]), (4, w[1])):
        bad, unsure = fp.codes_at_odds(kept[i], kept[i + 1], *ref.product(x.double(), weight.double()))
        assert bad == 0 and unsure < 0.05


@pytest.mark.parametrize("tokens,dim,out,left", SIZES)
def test_linear_8bit(tokens, dim, out, left):
    from paper_2609_21594_b200 import functional as F

    x, w, *_ = make(tokens, dim, out, left)
    dy = make(tokens, out, 8, left)[0] * 1e-3
    w8 = F.quantize(w, 128)
    y, *x8 = F.linear_8bit_forward(x, *w8)
    xv, wv = ref.unpack(x8[0].float(), x8[1], 1), ref.unpack(w8[0].float(), w8[1], 128)
    assert fp.excess(y, xv @ wv.T) <= fp.LIMIT
    dx, dw = F.linear_8bit_backward(dy, *x8, *w8)
    assert fp.excess(dx, ref.unpack(*ref.pack(dy, 1), 1) @ wv) <= fp.LIMIT
    assert fp.excess(dw, dy.double().T @ xv) <= fp.LIMIT
