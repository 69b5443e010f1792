"""What the differentiable operators keep for their backward pass, with a stand-in for the rotation so that no GPU is needed."""
import numpy as np
import pytest
import torch


def turned(tensors, inv_freq, layout="half", amplitude=1.0, positions=None, offset=0, inverse=False, out=None):
    """A rotation of one pair per head, on the CPU."""
    angle = (positions.double() + offset) * float(np.asarray(inv_freq)[0]) * (-1 if inverse else 1)
    c, s = angle.cos()[..., None], angle.sin()[..., None]
    return tuple(torch.stack((x[..., 0] * c - x[..., 1] * s, x[..., 0] * s + x[..., 1] * c), -1).to(x.dtype) for x in tensors)


@pytest.fixture
def rotary(monkeypatch):
    from paper_2609_21594_b200 import functional as F

    monkeypatch.setattr(F, "rotary_forward", turned)
    return F.rotary


def test_positions_written_before_the_backward_pass_are_an_error(rotary):
    x = torch.randn(1, 5, 1, 2, dtype=torch.float64, requires_grad=True)
    positions = torch.arange(5, dtype=torch.int32)[None]
    y, = rotary([x], np.array([0.3]), positions=positions)
    positions.copy_(torch.arange(5, 10, dtype=torch.int32)[None])      # the next micro-batch
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.sum().backward()


def test_frequencies_changed_before_the_backward_pass_do_not_count(rotary):
    x = torch.randn(1, 5, 1, 2, dtype=torch.float64, requires_grad=True)
    positions, f = torch.arange(5, dtype=torch.int32)[None], np.array([0.3])
    y, = rotary([x], f, positions=positions)
    f[0] = 7.0
    c = torch.randn(y.shape, dtype=torch.float64)
    y.backward(c)
    want, = turned([c], np.array([0.3]), positions=positions, inverse=True)
    assert torch.allclose(x.grad, want, rtol=1e-12, atol=1e-12)
