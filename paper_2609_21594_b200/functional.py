"""torch front end of the layer operators: layer norm, rotary positions, attention, the gated feed-forward block and the 8-bit linear layer, forward
and backward.

What a training program needs around the matrices that `optim.Muon` updates.  The `*_forward` / `*_backward` pairs are defined in
`csrc/front.cpp` (argument checks and marshalling, built as `_front`) and their arithmetic runs in the CUDA library, on the current
stream of the tensors' device.  `layer_norm`, `rotary`, `attention`, `feed_forward` and `linear_8bit` are differentiable; the pairs are the same calls for programs that
keep their own tape.  Each host thread has a context of its own per device (autograd calls backward passes from another thread); all
of a device's record an expired wait in one word, which `synchronize_and_check` reads.
A thread's first call on a device makes its context, which allocates: calls are captured into a graph after one ordinary call.
"""
from __future__ import annotations

import ctypes as C
from typing import Optional, Sequence, Tuple

import numpy as np
import torch

from . import binding as mb  # first: it loads the library that _front is linked with

try:
    from . import _front
except ImportError as e:
    raise ImportError("the torch front end of the layer operators (_front.so) is missing or does not fit this torch: build it with "
                      "`python -m paper_2609_21594_b200.build`, which needs a C++ compiler and the headers of Python and torch") from e
from ._front import attention_backward, attention_forward, layer_norm_backward, layer_norm_forward, rotary_forward  # noqa: F401
from ._front import dequantize, feed_forward_backward, feed_forward_forward, linear_8bit_backward, linear_8bit_forward, quantize  # noqa: F401
from .binding import muon_rotary_frequencies as rotary_frequencies  # noqa: F401  (part of this module's interface)


def _refused(code: int, where: str) -> None:
    raise mb.MuonError(code, where)


_front.set_refused(_refused)


class _ThreadContext(mb.Context):
    """A context that belongs to its thread: closing this object leaves it."""

    def __init__(self, address: int):
        self.opt, self.handle, self._ws = mb.muon_default_options(), C.c_void_p(address), None

    def close(self) -> None:
        pass


def context(device: Optional[torch.device] = None) -> mb.Context:
    """This thread's context of a device (default: the current one): the one the functions of this module use there."""
    return _ThreadContext(_front.context(torch.cuda.current_device() if device is None or device.index is None else device.index))


def synchronize_and_check(device: Optional[torch.device] = None) -> None:
    """Synchronises the device (default: the current one) and raises MuonError (ERR_DEVICE_TIMEOUT) when a bounded wait of a call of this module
    has expired there, from whatever thread: that call's results are incomplete.  The word stays set until
    `context(device).muon_clear_device_status()`."""
    index = torch.cuda.current_device() if device is None or device.index is None else device.index
    torch.cuda.synchronize(index)
    with torch.cuda.device(index):
        code = context(torch.device("cuda", index)).muon_synchronize_and_check()
    if code != mb.OK:
        raise mb.MuonError(code, "muon_synchronize_and_check")


def _heads(t: torch.Tensor) -> mb.Heads:
    """The descriptor of a 4-D tensor as an object, for calls of the binding's Context."""
    s = t.stride()
    return mb.Heads(t.data_ptr(), s[0], s[1], s[2])


class _LayerNorm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, bias, eps, center):
        y, mean, rstd = layer_norm_forward(x, weight, bias, eps, center)
        ctx.save_for_backward(x, weight, mean, rstd)
        ctx.bias_dtype = None if bias is None else bias.dtype
        return y

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dy):
        x, weight, mean, rstd = ctx.saved_tensors
        dx, dw, db = layer_norm_backward(dy, x, weight, mean, rstd, ctx.bias_dtype is not None and ctx.needs_input_grad[2], ctx.bias_dtype)
        return dx, dw, db, None, None


def layer_norm(x: torch.Tensor, weight: Optional[torch.Tensor] = None, bias: Optional[torch.Tensor] = None, eps: float = 1e-5,
               center: bool = True) -> torch.Tensor:
    """Differentiable layer norm (center=False: RMS norm) over the last dimension."""
    return _LayerNorm.apply(x, weight, bias, eps, center)


class _Rotary(torch.autograd.Function):
    @staticmethod
    def forward(ctx, inv_freq, layout, amplitude, positions, offset, *tensors):
        inv_freq = np.asarray(inv_freq, dtype=np.float64).copy()      # the caller may change its own before the backward pass
        ctx.save_for_backward(positions)                     # watched: autograd refuses a backward pass after they were written
        ctx.args = (inv_freq, layout, amplitude, offset)
        return rotary_forward(tensors, inv_freq, layout, amplitude, positions, offset)

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, *grads):
        inv_freq, layout, amplitude, offset = ctx.args
        positions, = ctx.saved_tensors
        return (None,) * 5 + rotary_forward(grads, inv_freq, layout, amplitude, positions, offset, inverse=True)


def rotary(tensors: Sequence[torch.Tensor], inv_freq, layout: str = "half", amplitude: float = 1.0,
           positions: Optional[torch.Tensor] = None, offset: int = 0) -> Tuple[torch.Tensor, ...]:
    """Differentiable `rotary_forward`.  The backward pass turns by the same angles: positions written in between are an error, inv_freq is copied."""
    return _Rotary.apply(inv_freq, layout, amplitude, positions, offset, *tensors)


class _Attention(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, v, causal, window, scale, q_lens, k_lens, q_offsets, k_offsets):
        o, lse = attention_forward(q, k, v, causal, window, scale, q_lens, k_lens, q_offsets, k_offsets)
        ctx.save_for_backward(q, k, v, o, lse, q_lens, k_lens, q_offsets, k_offsets)
        ctx.mask = (causal, window, scale)
        return o

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, do):
        q, k, v, o, lse, *lens = ctx.saved_tensors
        return attention_backward(do, q, k, v, o, lse, *ctx.mask, *lens) + (None,) * 7


def attention(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, causal: bool = True, window: int = 0, scale: Optional[float] = None,
              q_lens: Optional[torch.Tensor] = None, k_lens: Optional[torch.Tensor] = None,
              q_offsets: Optional[torch.Tensor] = None, k_offsets: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Differentiable `attention_forward`: o alone."""
    return _Attention.apply(q, k, v, causal, window, scale, q_lens, k_lens, q_offsets, k_offsets)


class _FeedForward(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, w_gate, w_up, w_down, activation, checkpoint):
        y, kept = feed_forward_forward(x, w_gate, w_up, w_down, activation, checkpoint)
        ctx.save_for_backward(x if checkpoint == "full" else None, w_gate, w_up, w_down, *kept)
        ctx.activation = activation
        return y

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dy):
        x, w_gate, w_up, w_down, *kept = ctx.saved_tensors
        return feed_forward_backward(dy, x, w_gate, w_up, w_down, kept, ctx.activation, ctx.needs_input_grad[:4]) + (None, None)


def feed_forward(x: torch.Tensor, w_gate: torch.Tensor, w_up: torch.Tensor, w_down: torch.Tensor, activation: str = "silu",
                 checkpoint: str = "full") -> torch.Tensor:
    """Differentiable `feed_forward_forward`: y alone.  checkpoint: "full" or "8bit"; where nothing asks for gradients nothing is kept.
    The products are made for bf16.  In fp32 they run on CUDA cores, about half as fast as torch's where there is much to multiply."""
    if checkpoint not in ("full", "8bit"):
        raise ValueError("checkpoint is 'full' or '8bit'")
    if not (torch.is_grad_enabled() and any(t.requires_grad for t in (x, w_gate, w_up, w_down))):
        return feed_forward_forward(x, w_gate, w_up, w_down, activation, "none")[0]
    return _FeedForward.apply(x, w_gate, w_up, w_down, activation, checkpoint)


class _Linear8bit(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight):
        w_codes, w_scales = quantize(weight, 128)
        y, x_codes, x_scales = linear_8bit_forward(x, w_codes, w_scales)
        ctx.save_for_backward(x_codes, x_scales, w_codes, w_scales)
        ctx.dtype = weight.dtype
        return y

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dy):
        # dw comes rounded to bf16, as dy and x are, and an fp32 weight is given it as that: dy's own rounding moves it by as much
        dx, dw = linear_8bit_backward(dy, *ctx.saved_tensors, ctx.needs_input_grad)
        return dx, None if dw is None else dw.to(ctx.dtype)


def linear_8bit(x: torch.Tensor, weight: torch.Tensor) -> torch.Tensor:
    """Differentiable x weight' whose products are formed in 8 bits (`linear_8bit_forward`, `linear_8bit_backward`): bf16 x [..., dim], bf16 or fp32
    weight [out, dim], whose gradient is rounded to bf16 in either case.  Keeps x and the weight in 8 bits for the backward pass.  The gradient of the rounding to
    8 bits is taken as 1.  Every call packs the weight: a program that multiplies with one weight many times packs it once and calls `linear_8bit_forward`."""
    return _Linear8bit.apply(x, weight)
