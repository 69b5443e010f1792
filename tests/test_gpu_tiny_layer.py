"""The example that runs the layer operators and the Muon step together: it learns, it repeats, and its gradients are those of the same
layer written out in 64 bits."""
import importlib.util
import math
import os
import subprocess
import sys

import pytest
import torch

import layer_reference as ref

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def example():
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "tiny_layer.py")
    spec = importlib.util.spec_from_file_location("tiny_layer", path)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def test_it_learns_and_repeats():
    t = example()
    losses = t.train(200)
    guess = math.log(t.VOCAB)
    assert 0.8 * guess < losses[0] < 1.3 * guess and all(math.isfinite(x) for x in losses)
    assert sum(losses[-10:]) / 10 < guess / 3
    assert t.train(3) == losses[:3]


def test_gradients_against_the_layer_in_64_bits():
    """Every activation is rounded to bf16 (2^-8) a few times on the way there and back, independently: the gradient of a matrix is off by a few
    times 2^-8 of its norm at most.  2^-4 of the norm leaves room for that and none for a wrong term."""
    t = example()
    g = torch.Generator(device="cuda").manual_seed(3)
    model = t.TinyLayer(g)
    tokens, positions, offsets, learn = t.batch(g, documents=3)
    torch.nn.functional.cross_entropy(model(tokens, positions, offsets)[learn], tokens[learn + 1]).backward()

    p = {n: w.detach().double().requires_grad_() for n, w in model.named_parameters()}
    norm = lambda x, i: ref.norm_of(x, p[f"norms.{i}"], p[f"biases.{i}"], 1e-5)  # noqa: E731
    x = p["embedding"][tokens]
    h = norm(x, 0)
    q, k, v = ((h @ p[w].T).view(-1, t.HEADS, t.DIM // t.HEADS) for w in ("wq", "wk", "wv"))
    f = torch.as_tensor(model.inv_freq, device="cuda")
    angle = positions.double()[:, None, None] * f
    rotate = lambda z: torch.cat((z[..., :32] * angle.cos() - z[..., 32:] * angle.sin(), z[..., :32] * angle.sin() + z[..., 32:] * angle.cos()), -1)  # noqa: E731
    s = torch.einsum("qhd,khd->hqk", rotate(q), rotate(k)) / math.sqrt(q.shape[-1])
    i = torch.arange(len(tokens), device="cuda")
    doc = (i[:, None] >= offsets[None, 1:]).sum(-1)
    s = s.masked_fill((doc[:, None] != doc[None]) | (i[:, None] < i[None]), -math.inf)
    x = x + torch.einsum("hqk,khd->qhd", s.softmax(-1), v).reshape(-1, t.DIM) @ p["wo"].T
    x = x + torch.relu(norm(x, 1) @ p["up"].T) @ p["down"].T
    torch.nn.functional.cross_entropy((norm(x, 2) @ p["embedding"].T)[learn], tokens[learn + 1]).backward()
    for n, w in model.named_parameters():
        off = float((w.grad.double() - p[n].grad).norm() / p[n].grad.norm())
        assert off <= 2.0 ** -4, (n, off)


_EXIT = """
import threading, torch
from paper_2609_21594_b200 import functional as F
x = torch.randn(1, 32, 4, 64, device="cuda", dtype=torch.bfloat16, requires_grad=True)
F.attention(x, x, x).sum().backward()
seen = []
def other():
    F.layer_norm_forward(torch.ones(4, 8, device="cuda"))
    seen.append(F.context().handle.value)
for _ in range(3):
    t = threading.Thread(target=other)
    t.start()
    t.join()
torch.cuda.synchronize()
assert seen[0] != F.context().handle.value and len(set(seen)) == 1
assert F.context().muon_last_device_status() == 0
"""


def test_threads_end_and_the_process_exits():
    """A thread's context passes to the next one, and threads that end while the process exits (autograd's) do not call into the device."""
    for _ in range(3):
        r = subprocess.run([sys.executable, "-c", _EXIT], cwd=ROOT, capture_output=True, text=True, timeout=300)
        assert r.returncode == 0, r.stderr[-2000:]
