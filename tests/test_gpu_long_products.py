"""Products that keep the device busy for a long time: a bounded wait is for what does not come, not for what takes long."""
import pytest
import torch

import feed_forward_reference as ref

pytestmark = pytest.mark.gpu


def test_a_launch_of_half_a_second_reports_no_expired_wait():
    """57344 tokens of 57344 x 57344: 0.45 s in the gated product alone, 40 GB.  Some rows of the result against 64 bits."""
    from paper_2609_21594_b200 import functional as F

    n = 57344
    if torch.cuda.mem_get_info()[0] < 50e9:
        pytest.skip("50 GB of free memory are needed")
    F.synchronize_and_check()
    g = torch.Generator(device="cuda").manual_seed(0)
    x, *w = (torch.empty((n, n), dtype=torch.bfloat16, device="cuda").normal_(0, s, generator=g) for s in (1, n ** -0.5, n ** -0.5, n ** -0.5))
    y, _ = F.feed_forward_forward(x, *w, "silu", "none")
    torch.cuda.synchronize()
    expired = F.context().muon_last_device_status()
    F.context().muon_clear_device_status()                   # the word is every later call's, too
    assert expired == 0
    rows = torch.tensor([0, 1, 255, 256, 31000, n - 1], device="cuda")
    cut = lambda a, b: torch.cat([a @ b[i:i + 4096].double().T for i in range(0, n, 4096)], 1)  # noqa: E731
    xr = x[rows].double()
    h = (ref.act(cut(xr, w[0]), "silu") * cut(xr, w[1])).bfloat16().double()
    value = cut(h, w[2])
    # the result's rounding and what fp32 sums turn in those of h, beside which a tile that was left out stands out
    assert float((y[rows].double() - value).norm() / value.norm()) < 2 * ref.half(torch.bfloat16)
    del x, w, y
    torch.cuda.empty_cache()


def squares(a):
    return float((a * a).sum())


def check_long_sum(got, parts):
    """`parts`: pairs of 64-bit factors, a few tokens at a time.  Off by the result's rounding and little else: sums that are cut instead of rounded may add a
    fifth of it to the norm's square (2^18 terms of random sign: a twentieth), where those of 2^21 terms in one piece add twice of it."""
    value = sum(a().T @ b() for a, b in parts)
    alone = squares(value.to(got.dtype).double() - value)
    assert squares(got.double() - value) <= 1.2 * alone


@pytest.mark.parametrize("keep", ["full", "8bit"])
@pytest.mark.parametrize("tokens,dim,hidden", [((1 << 21) + 77, 64, 136), ((1 << 21) + 1, 50, 72), (1 << 20, 72, 264)])
def test_sums_over_many_tokens(tokens, dim, hidden, keep):
    from paper_2609_21594_b200 import functional as F

    g = torch.Generator(device="cuda").manual_seed(0)
    x, dy = (torch.empty((tokens, dim), device="cuda").normal_(0, 1, generator=g).bfloat16() for _ in range(2))
    w = [torch.empty(s, device="cuda").normal_(0, s[1] ** -0.5, generator=g).bfloat16() for s in ((hidden, dim), (hidden, dim), (dim, hidden))]
    _, kept = F.feed_forward_forward(x, *w, "silu", keep)
    _, *got = F.feed_forward_backward(dy, x if keep == "full" else None, *w, kept)

    def piece(i):                                            # (dg, du, h, x, dy) of some tokens, rounded as documented
        at = slice(i, i + (1 << 18))
        xi, gi, ui = (x[at].double(), kept[0][at].double(), kept[1][at].double()) if keep == "full" else (
            ref.unpack(kept[k][at].float(), kept[k + 1][at], 1) for k in (0, 2, 4))
        a, slope = ref.act_and_slope(gi, "silu")
        dh = dy[at].double() @ w[2].double()
        return [t.bfloat16().double() for t in (dh * ui * slope, dh * a, a * ui)] + [xi.bfloat16().double(), dy[at].double()]

    starts = range(0, tokens, 1 << 18)
    for k, (a, b) in enumerate(((0, 3), (1, 3), (4, 2))):
        check_long_sum(got[k], [(lambda i=i: piece(i)[a], lambda i=i: piece(i)[b]) for i in starts])
        need = [False] + [i == k for i in range(3)]
        assert torch.equal(F.feed_forward_backward(dy, x if keep == "full" else None, *w, kept, "silu", need)[k + 1], got[k])
    F.synchronize_and_check()


def test_sums_over_many_tokens_of_the_8_bit_layer():
    from paper_2609_21594_b200 import functional as F

    tokens, dim, out = (1 << 21) + 77, 64, 136
    g = torch.Generator(device="cuda").manual_seed(0)
    x, dy = (torch.empty((tokens, n), device="cuda").normal_(0, 1, generator=g).bfloat16() for n in (dim, out))
    w8 = F.quantize(torch.empty((out, dim), device="cuda").normal_(0, 1, generator=g), 128)
    _, *x8 = F.linear_8bit_forward(x, *w8)
    _, dw = F.linear_8bit_backward(dy, *x8, *w8)
    starts = range(0, tokens, 1 << 18)
    cut = lambda i: slice(i, i + (1 << 18))  # noqa: E731
    check_long_sum(dw, [(lambda i=i: dy[cut(i)].double(), lambda i=i: ref.unpack(x8[0][cut(i)].float(), x8[1][cut(i)], 1)) for i in starts])


def test_a_row_too_long_for_the_tensor_cores():
    """dim = 2^21: sums that the tensor cores would cut by as much as the result's rounding, on CUDA cores."""
    from paper_2609_21594_b200 import functional as F

    n = 1 << 21
    g = torch.Generator(device="cuda").manual_seed(0)
    x, wg, wu = (torch.empty((r, n), device="cuda").normal_(0, s, generator=g).bfloat16() for r, s in ((40, 1), (64, n ** -0.5), (64, n ** -0.5)))
    wd = torch.zeros((n, 64), dtype=torch.bfloat16, device="cuda")
    _, (gate, up) = F.feed_forward_forward(x, wg, wu, wd)
    for got, w in ((gate, wg), (up, wu)):
        check_long_sum(got, [(lambda i=i: x[:, i:i + (1 << 18)].double().T, lambda i=i, w=w: w[:, i:i + (1 << 18)].double().T) for i in range(0, n, 1 << 18)])


def test_long_sums_in_a_graph_on_another_stream_and_off_the_alignment():
    from paper_2609_21594_b200 import functional as F

    tokens, dim, hidden = (1 << 19) + 130, 40, 56
    g = torch.Generator(device="cuda").manual_seed(1)
    r = lambda *s: torch.empty(s, device="cuda").normal_(0, 1, generator=g).bfloat16()  # noqa: E731
    inputs = [[r(tokens, dim), r(tokens, dim), r(tokens, hidden), r(tokens, hidden)] for _ in range(2)]          # dy, x, gate, up
    w = [r(hidden, dim), r(hidden, dim), r(dim, hidden)]
    call = lambda dy, x, gate, up: F.feed_forward_backward(dy, x, *w, [gate, up])  # noqa: E731
    wants = [call(*i) for i in inputs]
    given = [t.clone() for t in inputs[0]]
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        call(*given)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        out = call(*given)
    for k in (1, 0, 1):
        for to, t in zip(given, inputs[k]):
            to.copy_(t)
        graph.replay()
        assert all(torch.equal(a, b) for a, b in zip(out, wants[k]))
    # rows that begin one element off: CUDA cores, whose sums have no parts
    wide = [torch.cat([t[:, :1], t, t[:, :1].expand(-1, 8 - 1)], 1)[:, 1:1 + t.shape[1]] for t in inputs[0]]
    starts = range(0, tokens, 1 << 18)
    for a, b in zip(call(*wide)[1:], wants[0][1:]):
        assert float((a.double() - b.double()).norm() / b.double().norm()) < ref.half(torch.bfloat16)      # both are rounded once, most of them alike
    dy = inputs[0][0]
    cut = lambda t, i: t[i:i + (1 << 18)].double()  # noqa: E731
    products = [(lambda i=i: cut(dy, i), lambda i=i: (ref.act(cut(inputs[0][2], i), "silu") * cut(inputs[0][3], i)).bfloat16().double()) for i in starts]
    check_long_sum(wants[0][3], products)
    check_long_sum(call(*wide)[3], products)
    F.synchronize_and_check()
