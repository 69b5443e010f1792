"""The differentiable rotation on the device: what it keeps between forward and backward."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu


def test_positions_and_frequencies_between_forward_and_backward():
    from paper_2609_21594_b200 import functional as F

    x = torch.randn(2, 33, 4, 64, device="cuda", requires_grad=True)
    c = torch.randn(x.shape, device="cuda")
    positions = torch.arange(66, dtype=torch.int32, device="cuda").view(2, 33)
    f = 10000.0 ** (-np.arange(32) / 32)
    want, = F.rotary_forward([c], f, positions=positions, inverse=True)
    y, = F.rotary([x], f, positions=positions)
    f *= 3
    y.backward(c)
    assert torch.equal(x.grad, want)
    y, = F.rotary([x], f, positions=positions)
    positions += 7
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.backward(c)


def test_without_positions():
    from paper_2609_21594_b200 import functional as F

    x = torch.randn(1, 33, 4, 64, device="cuda", requires_grad=True)
    c = torch.randn(x.shape, device="cuda")
    f = 10000.0 ** (-np.arange(32) / 32)
    y, = F.rotary([x], torch.from_numpy(f), offset=5)
    y.backward(c)
    want, = F.rotary_forward([c], list(f), offset=5, inverse=True)
    assert torch.equal(x.grad, want)
