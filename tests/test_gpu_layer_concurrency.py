"""The layer operators captured into a graph, and called from two threads on two streams at once."""
import threading

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

FREQ = 10000.0 ** (-np.arange(32) / 32)


def inputs(seed, n=300, heads=4, dtype=torch.bfloat16):
    g = torch.Generator(device="cuda").manual_seed(seed)
    r = lambda *s: torch.randn(s, generator=g, device="cuda").to(dtype)  # noqa: E731
    return r(1, n, heads, 64), r(1, n, heads // 2, 64), r(1, n, heads // 2, 64), r(1, n, heads, 64), r(n, 256)


def layer(q, k, v, do, x):
    """Every operator, forward and backward."""
    from paper_2609_21594_b200 import functional as F

    w = torch.ones(x.shape[1], device="cuda")
    q, k = F.rotary_forward((q, k), FREQ)
    o, lse = F.attention_forward(q, k, v)
    dq, dk, dv = F.attention_backward(do, q, k, v, o, lse)
    dq, dk = F.rotary_forward((dq, dk), FREQ, inverse=True)
    y, mean, rstd = F.layer_norm_forward(x, w, w)
    return (o, lse, dq, dk, dv, y) + F.layer_norm_backward(y, x, w, mean, rstd)


@pytest.mark.parametrize("n,dtype", [(64, torch.bfloat16), (300, torch.bfloat16), (1000, torch.bfloat16), (300, torch.float32)])
def test_graph(n, dtype):
    """Captured once, replayed on new inputs: the bits of ordinary calls.  The first call of a thread makes its context, so one comes before."""
    static = inputs(0, n, dtype=dtype)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        layer(*static)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = layer(*static)
    for seed in (1, 2, 3):
        fresh = inputs(seed, n, dtype=dtype)
        for a, b in zip(static, fresh):
            a.copy_(b)
        graph.replay()
        graph.replay()
        for a, b in zip(captured, layer(*fresh)):
            assert torch.equal(a, b)


def test_graph_of_a_training_step():
    from paper_2609_21594_b200 import functional as F

    q, k, v, do, x = inputs(5)
    w = torch.ones(256, device="cuda", requires_grad=True)
    q, k, v, x = (t.requires_grad_() for t in (q, k, v, x))
    leaves = [q, k, v, x, w]

    def step():
        for t in leaves:
            t.grad = None
        a, b = F.rotary((q, k), FREQ)
        (F.attention(a, b, v) * do).sum().backward()
        (F.layer_norm(x, w) ** 2).sum().backward()

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
        step()
    torch.cuda.current_stream().wait_stream(side)
    want = [t.grad.clone() for t in leaves]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for _ in range(2):
        for t in leaves:
            t.grad.fill_(float("nan"))
        graph.replay()
        assert all(torch.equal(t.grad, g) for t, g in zip(leaves, want))


def test_two_threads_on_two_streams():
    sets = [inputs(i, n) for i, n in ((10, 300), (11, 513))]
    want = [layer(*s) for s in sets]
    torch.cuda.synchronize()
    wrong = []

    def work(i):
        stream = torch.cuda.Stream()
        with torch.cuda.stream(stream):
            for _ in range(30):
                got = layer(*sets[i])
                if not all(torch.equal(a, b) for a, b in zip(got, want[i])):
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
