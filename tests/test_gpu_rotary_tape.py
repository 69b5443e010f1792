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


def test_what_is_written_in_place_is_seen_by_autograd():
    from paper_2609_21594_b200 import functional as F

    f = 10000.0 ** (-np.arange(32) / 32)
    x, w = torch.randn(1, 8, 2, 64, device="cuda"), torch.randn(1, 8, 2, 64, device="cuda", requires_grad=True)
    y = (w * x).sum()                                    # saves x
    version = x._version
    F.rotary_forward([x], f, out=[x])
    assert x._version == version + 1
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.backward()
    z = w * 1.0
    for out in (w, z, z[:, :, :, :]):
        before = out.detach().clone()
        with pytest.raises(ValueError):
            F.rotary_forward([x], f, out=[out])
        assert torch.equal(out.detach(), before)
    with torch.no_grad():
        F.rotary_forward([x], f, out=[w])
    assert torch.equal(w.detach(), F.rotary_forward([x], f)[0])
    with torch.inference_mode():
        a = torch.randn(1, 8, 2, 64, device="cuda")
        b = F.rotary_forward([a], f)[0]
        F.rotary_forward([a], f, out=[a])
        assert torch.equal(a, b)
