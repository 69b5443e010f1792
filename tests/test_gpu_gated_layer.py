"""The example that runs all layer operators together, and runs of the feed-forward block and the 8-bit linear layer as programs use them: in graphs,
on two streams at once, behind one another, over tensors of more than 2^31 elements."""
import importlib.util
import math
import os
import sys
import threading

import pytest
import torch

import feed_forward_reference as ff
import layer_reference as ref

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def example():
    folder = os.path.join(ROOT, "examples")
    sys.path.insert(0, folder)
    try:
        spec = importlib.util.spec_from_file_location("gated_layer", os.path.join(folder, "gated_layer.py"))
        module = importlib.util.module_from_spec(spec)
        spec.loader.exec_module(module)
        return module
    finally:
        sys.path.remove(folder)


@pytest.mark.parametrize("eight", [True, False])
def test_it_runs_and_repeats(eight):
    t = example()
    losses = t.train(4, eight=eight)
    assert all(math.isfinite(x) for x in losses) and 0.7 * math.log(t.VOCAB) < losses[0] < 1.4 * math.log(t.VOCAB)
    assert t.train(4, eight=eight) == losses


def test_gradients_against_the_layer_in_64_bits():
    """In bf16, where every activation is rounded (2^-8) a few times on the way there and back, independently: the gradient of a matrix is off by a few times
    2^-8 of its norm at most.  2^-4 of the norm leaves room for that and none for a wrong term."""
    t = example()
    g = torch.Generator(device="cuda").manual_seed(3)
    model = t.GatedLayer(g, eight=False)
    tokens, positions, offsets, learn = t.batch(g, documents=3)
    torch.nn.functional.cross_entropy(model(tokens, positions, offsets)[learn], tokens[learn + 1]).backward()

    p = {n: w.detach().double().requires_grad_() for n, w in model.named_parameters()}
    norm = lambda x, i: x / torch.sqrt((x * x).mean(-1, keepdim=True) + 1e-5) * p[f"norms.{i}"]  # noqa: E731
    x = p["embedding"][tokens]
    h = norm(x, 0)
    q, k, v = ((h @ p[w].T).view(len(tokens), -1, t.HEAD) for w in ("wq", "wk", "wv"))
    angle = positions.double()[:, None, None] * torch.as_tensor(model.inv_freq, device="cuda")
    rotate = lambda z: torch.cat((z[..., :32] * angle.cos() - z[..., 32:] * angle.sin(), z[..., :32] * angle.sin() + z[..., 32:] * angle.cos()), -1)  # noqa: E731
    k, v = (z.repeat_interleave(t.HEADS // t.KV_HEADS, 1) for z in (rotate(k), v))
    s = torch.einsum("qhd,khd->hqk", rotate(q), k) / math.sqrt(t.HEAD)
    i = torch.arange(len(tokens), device="cuda")
    doc = (i[:, None] >= offsets[None, 1:]).sum(-1)
    s = s.masked_fill((doc[:, None] != doc[None]) | (i[:, None] < i[None]), -math.inf)
    x = x + torch.einsum("hqk,khd->qhd", s.softmax(-1), v).reshape(-1, t.DIM) @ p["wo"].T
    h = norm(x, 1)
    x = x + (ff.act(h @ p["gate"].T, "silu") * (h @ p["up"].T)) @ p["down"].T
    torch.nn.functional.cross_entropy((norm(x, 2) @ p["embedding"].T)[learn], tokens[learn + 1]).backward()
    for n, w in model.named_parameters():
        off = float((w.grad.double() - p[n].grad).norm() / p[n].grad.norm())
        assert off <= 2.0 ** -4, (n, off)


def inputs(seed, tokens, dim=256, hidden=512, dtype=torch.bfloat16):
    g = torch.Generator(device="cuda").manual_seed(seed)
    r = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
    return (r(tokens, dim).to(dtype), (r(hidden, dim) * dim ** -0.5).to(dtype), (r(hidden, dim) * dim ** -0.5).to(dtype),
            (r(dim, hidden) * hidden ** -0.5).to(dtype), r(tokens, dim).to(dtype))


def block(x, wg, wu, wd, dy):
    """The block with both ways of keeping, and a linear layer, forward and backward."""
    from paper_2609_21594_b200 import functional as F

    out = []
    for keep in ("full", "8bit"):
        y, kept = F.feed_forward_forward(x, wg, wu, wd, "gelu", keep)
        out += [y, *(t.float() for t in kept), *F.feed_forward_backward(dy, x if keep == "full" else None, wg, wu, wd, kept, "gelu")]
    if x.dtype == torch.bfloat16:
        w8 = F.quantize(wd.T, 128)                           # [hidden, dim], as the linear layer takes it
        y, *x8 = F.linear_8bit_forward(x, *w8)
        out += [y, *(t.float() for t in x8), *F.linear_8bit_backward(y, *x8, *w8), F.dequantize(*x8, torch.float32)]
    return out


@pytest.mark.parametrize("tokens,dtype", [(1, torch.bfloat16), (100, torch.bfloat16), (1200, torch.bfloat16), (100, torch.float32)])
def test_graph(tokens, dtype):
    """Captured once, replayed on new inputs: the bits of ordinary calls.  Two graphs replayed in turn do not disturb one another."""
    statics = [inputs(k, tokens, dtype=dtype) for k in range(2)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        block(*statics[0])
    torch.cuda.current_stream().wait_stream(side)
    graphs, captured = [], []
    for s in statics:
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            captured.append(block(*s))
    for seed in (5, 6):
        fresh = [inputs(seed + 10 * k, tokens, dtype=dtype) for k in range(2)]
        for s, f in zip(statics, fresh):
            for a, b in zip(s, f):
                a.copy_(b)
        for _ in range(2):
            for g in graphs:
                g.replay()
        for c, f in zip(captured, fresh):
            for a, b in zip(c, block(*f)):
                assert torch.equal(a, b)


def test_graph_of_a_training_step():
    from paper_2609_21594_b200 import functional as F

    x, wg, wu, wd, dy = inputs(3, 200)
    leaves = [t.requires_grad_() for t in (x, wg, wu, wd)]
    head = torch.randn(128, 256, device="cuda", requires_grad=True)

    def step():
        for t in leaves + [head]:
            t.grad = None
        (F.linear_8bit(F.feed_forward(*leaves, checkpoint="8bit"), head).float() ** 2).sum().backward()

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
        step()
    torch.cuda.current_stream().wait_stream(side)
    want = [t.grad.clone() for t in leaves + [head]]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for _ in range(2):
        for t in leaves + [head]:
            t.grad.fill_(float("nan"))
        graph.replay()
        assert all(torch.equal(t.grad, g) for t, g in zip(leaves + [head], want))


def test_two_threads_on_two_streams():
    sets = [inputs(i, n) for i, n in ((10, 60), (11, 700))]
    want = [block(*s) for s in sets]
    torch.cuda.synchronize()
    wrong = []

    def work(i):
        stream = torch.cuda.Stream()
        with torch.cuda.stream(stream):
            for _ in range(20):
                if not all(torch.equal(a, b) for a, b in zip(block(*sets[i]), want[i])):
                    wrong.append(i)
        stream.synchronize()

    threads = [threading.Thread(target=work, args=(i,)) for i in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not wrong
    from paper_2609_21594_b200 import functional as F

    F.synchronize_and_check()


def test_a_call_right_behind_what_it_reads():
    """Weights, tokens and kept activations written just before the call, on the same stream: nothing of the call starts on what was there before."""
    from paper_2609_21594_b200 import functional as F

    x, wg, wu, wd, dy = inputs(7, 8, 1024, 2816)
    other = inputs(8, 8, 1024, 2816)
    wants = []
    for s in ((x, wg, wu, wd, dy), other):
        y, kept = F.feed_forward_forward(*s[:4], "silu", "8bit")
        w8 = F.quantize(s[1], 128)
        wants.append([y, *F.feed_forward_backward(s[4], None, *s[1:4], kept), F.linear_8bit_forward(s[0], *w8)[0]])
    live = [t.clone() for t in other]
    for k in range(20):
        source, want = ((x, wg, wu, wd, dy), wants[0]) if k % 2 == 0 else (other, wants[1])
        for a, b in zip(live, source):
            a.copy_(b)
        y, kept = F.feed_forward_forward(*live[:4], "silu", "8bit")
        w8 = F.quantize(live[1], 128)
        got = [y, *F.feed_forward_backward(live[4], None, *live[1:4], kept), F.linear_8bit_forward(live[0], *w8)[0]]
        for t in live:
            t.fill_(float("nan"))
        assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_more_than_2_to_the_31_elements():
    """Rows at the far end, whose offsets pass 32 bits: the bits of the same rows alone (a row's result does not depend on the others), and the block's
    gradients of them against the definition."""
    from paper_2609_21594_b200 import functional as F

    g = torch.Generator(device="cuda").manual_seed(0)
    rows, cols, tail = 300000, 7680, 300
    x = torch.empty((rows, cols), dtype=torch.bfloat16, device="cuda")
    x[:-tail].fill_(1.0)
    x[-tail:] = torch.randn((tail, cols), generator=g, device="cuda").bfloat16()
    codes, scales = F.quantize(x)
    want, e = ff.pack(x[-tail:], 1)
    assert torch.equal(codes[-tail:].double(), want) and torch.equal(scales[-tail:].long(), e)
    assert torch.equal(F.dequantize(codes, scales, torch.bfloat16)[-tail:].double(), ff.unpack(want, e, 1))
    del codes, scales

    tokens, dim, hidden = 280000, 64, 7680
    _, wg, wu, wd, _ = inputs(1, 1, dim, hidden)
    x = x.view(-1)[:tokens * dim].view(tokens, dim)
    x[-tail:] = torch.randn((tail, dim), generator=g, device="cuda").bfloat16()
    y, kept = F.feed_forward_forward(x, wg, wu, wd)
    value = ff.feed_forward(x[-tail:], wg, wu, wd, "silu")
    assert ff.worst(y[-tail:], value["y"]) <= 1
    for got, name in zip(kept, ("gate", "up")):
        assert ff.worst(got[-tail:], (value[name][0], ff.rounded(*value[name], torch.bfloat16))) <= 1
    dy = torch.zeros((tokens, dim), dtype=torch.bfloat16, device="cuda")
    dy[-tail:] = torch.randn((tail, dim), generator=g, device="cuda").bfloat16()
    got = F.feed_forward_backward(dy, x, wg, wu, wd, kept)
    # the other rows have no gradient and add zeros to the weights', of which the sums' bound knows nothing: it is that of the tail's rows alone
    want = ff.feed_forward_backward(dy[-tail:], x[-tail:], kept[0][-tail:], kept[1][-tail:], wg, wu, wd, "silu")
    assert ff.worst(got[0][-tail:], want[0]) <= 1 and not got[0][:-tail].any()
    for a, b in zip(got[1:], want[1:]):
        assert ff.worst(a, b) <= 1


def test_c_calls_refuse_what_lies_over_something_else():
    from paper_2609_21594_b200 import binding as mb, functional as F

    x, wg, wu, wd, dy = inputs(2, 16, 64, 128)
    y, g, u = torch.empty_like(x), torch.empty(16, 128, device="cuda").bfloat16(), torch.empty(16, 128, device="cuda").bfloat16()
    rows = lambda t: mb.Rows(t.data_ptr(), t.shape[1])  # noqa: E731
    d = mb.FeedForwardDesc(mb.DTYPE_BF16, mb.ACTIVATION_SILU, mb.KEEP_FULL, 16, 64, 128)
    n = mb.muon_feed_forward_workspace_bytes(d, False)
    ws = torch.empty(max(n, mb.muon_feed_forward_workspace_bytes(d, True)) + 256, dtype=torch.uint8, device="cuda")
    kept = mb.FeedForwardKept(gate=rows(g), up=rows(u))
    c = F.context()

    def forward(**kw):
        a = dict(x=rows(x), w_gate=rows(wg), w_up=rows(wu), w_down=rows(wd), y=rows(y), kept=kept, workspace=ws.data_ptr(), workspace_bytes=n)
        a.update(kw)
        c.muon_feed_forward_forward(d, *a.values())

    forward()
    want, (wantg, wantu) = F.feed_forward_forward(x, wg, wu, wd)
    assert torch.equal(y, want) and torch.equal(g, wantg) and torch.equal(u, wantu)
    bad = [dict(y=rows(x)), dict(y=rows(wg)), dict(kept=mb.FeedForwardKept(gate=rows(g), up=rows(g))), dict(kept=mb.FeedForwardKept(gate=rows(wd), up=rows(u))),
           dict(kept=None), dict(workspace=x.data_ptr()), dict(x=None), dict(w_up=None), dict(y=mb.Rows(y.data_ptr(), 63)), dict(x=mb.Rows(x.data_ptr() + 1, 64)),
           dict(workspace=ws.data_ptr() + 128), dict(kept=mb.FeedForwardKept(gate=rows(g), up=mb.Rows(g.data_ptr() + 16, 128)))]
    for kw in bad:
        with pytest.raises(mb.MuonError) as e:
            forward(**kw)
        assert e.value.code == mb.ERR_INVALID_ARG, kw
    for kw in (dict(workspace=None), dict(workspace_bytes=n - 1)):
        with pytest.raises(mb.MuonError) as e:
            forward(**kw)
        assert e.value.code == mb.ERR_WORKSPACE_TOO_SMALL

    n = mb.muon_feed_forward_workspace_bytes(d, True)
    dx, dg, du, dd = torch.empty_like(x), torch.empty_like(wg), torch.empty_like(wu), torch.empty_like(wd)

    def backward(**kw):
        a = dict(dy=rows(dy), x=rows(x), w_gate=rows(wg), w_up=rows(wu), w_down=rows(wd), kept=kept, dx=rows(dx), dw_gate=rows(dg), dw_up=rows(du), dw_down=rows(dd),
                 workspace=ws.data_ptr(), workspace_bytes=n)
        a.update(kw)
        c.muon_feed_forward_backward(d, *a.values())

    backward()
    for a, b in zip((dx, dg, du, dd), F.feed_forward_backward(dy, x, wg, wu, wd, (g, u))):
        assert torch.equal(a, b)
    for kw in (dict(dx=rows(dy)), dict(dw_gate=rows(du)), dict(dw_down=rows(wd)), dict(dx=rows(g)), dict(x=None), dict(dy=None), dict(workspace=dg.data_ptr())):
        with pytest.raises(mb.MuonError) as e:
            backward(**kw)
        assert e.value.code == mb.ERR_INVALID_ARG, kw
    backward(dx=None, dw_gate=None, dw_up=None, dw_down=None)
    d.keep = mb.KEEP_NONE
    with pytest.raises(mb.MuonError):
        backward()
    # no tokens: what has rows of them may be NULL, and the weights' gradients are zeros
    for keep in (mb.KEEP_FULL, mb.KEEP_8BIT):
        d.keep, d.tokens = keep, 0
        for t in (dg, du, dd):
            t.fill_(7.0)
        forward(x=None, y=None, kept=None, workspace=None, workspace_bytes=0)
        backward(dy=None, x=None, dx=None, kept=None, workspace=None, workspace_bytes=0)
        assert not any(t.any() for t in (dg, du, dd))
    d.tokens = 16
    # a wider row of the result keeps what lies behind its columns
    d.keep = mb.KEEP_FULL
    wide = torch.full((16, 80), 7.0, device="cuda").bfloat16()
    forward(y=mb.Rows(wide.data_ptr(), 80), workspace_bytes=n)
    assert torch.equal(wide[:, :64], want) and (wide[:, 64:] == 7).all()
    F.synchronize_and_check()
