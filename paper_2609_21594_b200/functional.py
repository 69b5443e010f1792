"""torch front end of the layer operators: layer norm, rotary positions and attention, forward and backward.

What a training program needs around the matrices that `optim.Muon` updates.  Argument checks and marshalling only: the arithmetic runs
in the CUDA library, on the current stream of the tensors' device.  `layer_norm`, `rotary` and `attention` are differentiable;
the `*_forward` / `*_backward` pairs are the same calls for programs that keep their own tape.  Each host thread has a context
of its own per device (autograd calls backward passes from another thread).
"""
from __future__ import annotations

import ctypes as C
import struct
import threading
from typing import Optional, Sequence, Tuple

import numpy as np
import torch

from . import binding as mb
from .binding import muon_rotary_frequencies as rotary_frequencies  # noqa: F401  (part of this module's interface)

_DTYPES = {torch.bfloat16: mb.DTYPE_BF16, torch.float32: mb.DTYPE_FP32}
_current_device = torch.cuda.current_device
_raw_stream = torch._C._cuda_getCurrentRawStream         # the current stream's handle, without building a Stream object
# memory images of muon_norm_desc_t, muon_rotary_desc_t, muon_attention_desc_t and of runs of muon_heads_t / muon_rotary_item_t
_NORM, _ROTARY, _ATTENTION = struct.Struct("4iqfi"), struct.Struct("7ifQQq"), struct.Struct("9if2i4Q")
_HEADS = {n: struct.Struct(f"{'Q3q' * n}") for n in (4, 8)}
_ITEM = struct.Struct("Q3qQ3q2i")
_DESC_BYTES, _HEADS_BYTES, _MAX_PAIRS = 128, 32, 256
_norm_forward, _norm_backward, _rotary_call = mb.lib.muon_layer_norm_forward, mb.lib.muon_layer_norm_backward, mb.lib.muon_rotary
_attention_forward, _attention_backward = mb.lib.muon_attention_forward, mb.lib.muon_attention_backward
_local = threading.local()


class _Lane:
    """What one host thread uses on one device: a context, and memory that descriptors are packed into for the length of a call."""

    def __init__(self, index: int):
        with torch.cuda.device(index):
            self.ctx = mb.Context()
        self.handle = self.ctx.handle
        self.memory = C.create_string_buffer(_DESC_BYTES + 10 * _HEADS_BYTES)
        self.desc = C.addressof(self.memory)
        self.heads = [self.desc + _DESC_BYTES + i * _HEADS_BYTES for i in range(10)]
        self.freq = np.empty(_MAX_PAIRS, dtype=np.float64)
        self.freq_at = self.freq.ctypes.data


def _lane(index: int) -> _Lane:
    try:
        return _local.lanes[index]
    except (AttributeError, KeyError):
        if not hasattr(_local, "lanes"):
            _local.lanes = {}
        lane = _local.lanes[index] = _Lane(index)
        return lane


def context(device: Optional[torch.device] = None) -> mb.Context:
    """This thread's context of a device (default: the current one): the one the functions of this module use there."""
    return _lane(_current_device() if device is None or device.index is None else device.index).ctx


def _dtype(t: torch.Tensor, what: str) -> int:
    d = _DTYPES.get(t.dtype)
    if d is None:
        raise ValueError(f"{what} must be bf16 or fp32, not {t.dtype}")
    return d


def _on(t: torch.Tensor, *others: Optional[torch.Tensor]) -> int:
    """The index of the device that all the tensors are on."""
    index = t.get_device()
    if index < 0:
        raise ValueError("the layer operators take CUDA tensors (there is no CPU fallback)")
    for o in others:
        if o is not None and o.get_device() != index:
            raise ValueError(f"tensors on {o.device} and {t.device} in one call")
    return index


def _refused(code: int, where: str) -> None:
    raise mb.MuonError(code, where)


def _address(t: Optional[torch.Tensor]) -> int:
    return 0 if t is None else t.data_ptr()


# ------------------------------------------------------------------------------------------------ layer norm
def _rows(t: torch.Tensor, what: str) -> torch.Tensor:
    """[..., cols] as [rows, cols] with contiguous rows: a view where the strides allow one, else a copy."""
    if t.dim() < 1 or t.shape[-1] < 1:
        raise ValueError(f"{what} needs a last dimension of at least one element")
    r = t if t.dim() == 2 else t.reshape(-1, t.shape[-1])
    return r if (r.shape[1] == 1 or r.stride(1) == 1) and (r.shape[0] <= 1 or r.stride(0) >= r.shape[1]) else r.contiguous()


def _ld(r: torch.Tensor) -> int:
    return max(r.stride(0), r.shape[1]) if r.shape[0] > 1 else r.shape[1]


def _param(p: Optional[torch.Tensor], cols: int, what: str) -> Optional[torch.Tensor]:
    if p is None:
        return None
    if p.shape != (cols,):
        raise ValueError(f"{what} must have shape ({cols},), not {tuple(p.shape)}")
    return p.contiguous()


def layer_norm_forward(x: torch.Tensor, weight: Optional[torch.Tensor] = None, bias: Optional[torch.Tensor] = None, eps: float = 1e-5,
                       center: bool = True) -> Tuple[torch.Tensor, Optional[torch.Tensor], torch.Tensor]:
    """(y, mean, rstd) over the last dimension; center=False is RMS norm and gives mean = None.  mean, rstd: fp32, x.shape[:-1]."""
    index = _on(x, weight, bias)
    if index != _current_device():
        with torch.cuda.device(index):
            return layer_norm_forward(x, weight, bias, eps, center)
    r = _rows(x, "x")
    rows, cols = r.shape
    weight, bias = _param(weight, cols, "weight"), _param(bias, cols, "bias")
    if weight is not None and bias is not None and weight.dtype != bias.dtype:
        raise ValueError("weight and bias must have one dtype")
    p = weight if weight is not None else bias
    lane = _lane(index)
    _NORM.pack_into(lane.memory, 0, _dtype(x, "x"), mb.DTYPE_FP32 if p is None else _dtype(p, "weight and bias"), 1 if center else 0, cols, rows,
                    eps, 0)
    y = torch.empty_like(x, memory_format=torch.contiguous_format)
    stat = x.shape[:-1]
    mean = x.new_empty(stat, dtype=torch.float32) if center else None
    rstd = x.new_empty(stat, dtype=torch.float32)
    rc = _norm_forward(lane.handle, lane.desc, r.data_ptr(), _ld(r), _address(weight), _address(bias), y.data_ptr(), cols, _address(mean),
                       rstd.data_ptr(), _raw_stream(index))
    if rc:
        _refused(rc, "muon_layer_norm_forward")
    return y, mean, rstd


def layer_norm_backward(dy: torch.Tensor, x: torch.Tensor, weight: Optional[torch.Tensor], mean: Optional[torch.Tensor], rstd: torch.Tensor,
                        bias: bool = True, bias_dtype: Optional[torch.dtype] = None
                        ) -> Tuple[torch.Tensor, Optional[torch.Tensor], Optional[torch.Tensor]]:
    """(dx, dweight, dbias); dweight is None without a weight, dbias unless `bias`.  The gradients have the weight's dtype (without a
    weight: bias_dtype, fp32 by default)."""
    index = _on(x, dy, weight, mean, rstd)
    if index != _current_device():
        with torch.cuda.device(index):
            return layer_norm_backward(dy, x, weight, mean, rstd, bias, bias_dtype)
    if dy.shape != x.shape or dy.dtype != x.dtype:
        raise ValueError("dy must have the shape and dtype of x")
    if rstd.shape != x.shape[:-1] or (mean is not None and mean.shape != rstd.shape):
        raise ValueError("mean and rstd must have the shape of x without its last dimension")
    if rstd.dtype != torch.float32 or (mean is not None and mean.dtype != torch.float32):
        raise ValueError("mean and rstd must be fp32")
    r, g = _rows(x, "x"), _rows(dy, "dy")
    rows, cols = r.shape
    weight = _param(weight, cols, "weight")
    mean, rstd = None if mean is None else mean.contiguous(), rstd.contiguous()
    pt = weight.dtype if weight is not None else (bias_dtype or torch.float32)
    if pt not in _DTYPES:
        raise ValueError(f"gradients must be bf16 or fp32, not {pt}")
    lane = _lane(index)
    _NORM.pack_into(lane.memory, 0, _dtype(x, "x"), _DTYPES[pt], 0 if mean is None else 1, cols, rows, 0.0, 0)
    dx = torch.empty_like(x, memory_format=torch.contiguous_format)
    dw = torch.empty_like(weight) if weight is not None else None
    db = None if not bias else torch.empty_like(weight) if weight is not None else x.new_empty(cols, dtype=pt)
    n = mb.muon_layer_norm_workspace_bytes(lane.desc) if dw is not None or db is not None else 0
    ws = x.new_empty(n, dtype=torch.uint8) if n else None
    rc = _norm_backward(lane.handle, lane.desc, g.data_ptr(), _ld(g), r.data_ptr(), _ld(r), _address(weight), _address(mean), rstd.data_ptr(),
                        dx.data_ptr(), cols, _address(dw), _address(db), _address(ws), n, _raw_stream(index))
    if rc:
        _refused(rc, "muon_layer_norm_backward")
    return dx, dw, db


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


# ------------------------------------------------------------------------------------------------ strided [batch, tokens, heads, dim] tensors
def _heads4(t: torch.Tensor, what: str) -> torch.Tensor:
    """As [batch, tokens, heads, dim] with a contiguous last dimension (a copy only where it is not)."""
    if t.dim() == 3:
        t = t[None]
    elif t.dim() != 4:
        raise ValueError(f"{what} must be [batch, tokens, heads, dim] or [tokens, heads, dim]")
    return t if t.stride(3) == 1 or t.shape[3] == 1 else t.contiguous()


def _heads(t: torch.Tensor) -> mb.Heads:
    """The descriptor of a 4-D tensor as an object, for calls of the binding."""
    s = t.stride()
    return mb.Heads(t.data_ptr(), s[0], s[1], s[2])


def _like(t: torch.Tensor) -> torch.Tensor:
    return torch.empty_like(t, memory_format=torch.contiguous_format)


# ------------------------------------------------------------------------------------------------ rotary positions
def rotary_forward(tensors: Sequence[torch.Tensor], inv_freq, layout: str = "half", amplitude: float = 1.0,
                   positions: Optional[torch.Tensor] = None, offset: int = 0, inverse: bool = False,
                   out: Optional[Sequence[torch.Tensor]] = None) -> Tuple[torch.Tensor, ...]:
    """Turns up to four [batch, tokens, heads, dim] (or [tokens, heads, dim]) tensors that share positions, in one launch.

    inv_freq: host, fp64 radians per position of each pair (see `rotary_frequencies`); twice its length is the part of the head that is
    turned, the rest is copied.  layout: "half" (i with i + n/2) or "interleaved" (2i with 2i + 1).  positions: int32 [batch, tokens] on
    the device, else offset + 0, 1, 2...; offset is added to given positions too.  inverse turns back, which is the backward pass.
    out: tensors to write, which may be the inputs themselves."""
    count = len(tensors)
    if not 1 <= count <= 4:
        raise ValueError("one to four tensors")
    if layout != "half" and layout != "interleaved":
        raise ValueError("layout is 'half' or 'interleaved'")
    first = tensors[0]
    index = _on(first, positions, *tensors[1:])
    if index != _current_device():
        with torch.cuda.device(index):
            return rotary_forward(tensors, inv_freq, layout, amplitude, positions, offset, inverse, out)
    lane = _lane(index)
    dtype = first.dtype
    b, n, d = None, None, None
    at = _DESC_BYTES
    keep, res = [], []
    if out is not None and (len(out) != count or any(o.shape != t.shape or o.dtype != t.dtype or o.device != t.device for o, t in zip(out, tensors))):
        raise ValueError("out must match the tensors")
    for i, t in enumerate(tensors):
        x = _heads4(t, "a tensor")
        xb, xn, xh, xd = x.shape
        if b is None:
            b, n, d = xb, xn, xd
        elif xb != b or xn != n or xd != d or t.dtype != dtype:
            raise ValueError("the tensors must agree in batch, tokens, head size and dtype")
        if out is None:
            o = torch.empty_like(t, memory_format=torch.contiguous_format)
        else:
            o = out[i]
            if o.stride(-1) != 1 and xd > 1:
                raise ValueError("out must have a contiguous last dimension")
        s, u = x.stride(), o.stride()
        _ITEM.pack_into(lane.memory, at, x.data_ptr(), s[0], s[1], s[2], o.data_ptr(), u[0] if len(u) == 4 else 0, u[-3], u[-2], xh, 0)
        at += _ITEM.size
        keep.append(x)
        res.append(o)
    freq = np.asarray(inv_freq, dtype=np.float64)
    pairs = freq.size
    if freq.ndim != 1 or not 1 <= pairs <= d // 2 or pairs > _MAX_PAIRS:
        raise ValueError(f"inv_freq must hold one to {min(d // 2, _MAX_PAIRS)} frequencies for heads of {d}")
    lane.freq[:pairs] = freq
    if positions is not None:
        if positions.dtype != torch.int32 or positions.numel() != b * n:
            raise ValueError("positions must be int32, one for each token")
        positions = positions.contiguous()
    _ROTARY.pack_into(lane.memory, 0, _dtype(first, "the tensors"), 1 if layout == "interleaved" else 0, 1 if inverse else 0, d, 2 * pairs, b, n,
                      amplitude, lane.freq_at, _address(positions), offset)
    rc = _rotary_call(lane.handle, lane.desc, lane.desc + _DESC_BYTES, count, _raw_stream(index))
    if rc:
        _refused(rc, "muon_rotary")
    return tuple(res)


class _Rotary(torch.autograd.Function):
    @staticmethod
    def forward(ctx, inv_freq, layout, amplitude, positions, offset, *tensors):
        ctx.args = (inv_freq, layout, amplitude, positions, offset)
        return rotary_forward(tensors, inv_freq, layout, amplitude, positions, offset)

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, *grads):
        inv_freq, layout, amplitude, positions, offset = ctx.args
        return (None,) * 5 + rotary_forward(grads, inv_freq, layout, amplitude, positions, offset, inverse=True)


def rotary(tensors: Sequence[torch.Tensor], inv_freq, layout: str = "half", amplitude: float = 1.0,
           positions: Optional[torch.Tensor] = None, offset: int = 0) -> Tuple[torch.Tensor, ...]:
    """Differentiable `rotary_forward`."""
    return _Rotary.apply(inv_freq, layout, amplitude, positions, offset, *tensors)


# ------------------------------------------------------------------------------------------------ attention
def _int32(t: torch.Tensor, n: int, what: str) -> torch.Tensor:
    if t.dtype != torch.int32 or t.dim() != 1 or t.numel() != n:
        raise ValueError(f"{what} must be a 1-D int32 tensor of {n}")
    return t.contiguous()


def _attention_call(lane: _Lane, q, k, v, causal, window, scale, q_lens, k_lens, q_offsets, k_offsets):
    """Packs the descriptor; gives q, k, v as 4-D tensors, and the tensors that the descriptor points into, to be kept for the call."""
    packed = q_offsets is not None or k_offsets is not None
    dims = 3 if packed else 4
    if q.dim() != dims or k.dim() != dims or v.dim() != dims:
        raise ValueError("q, k, v are [batch, tokens, heads, dim], or [tokens, heads, dim] with offsets")
    if q.dtype != k.dtype or q.dtype != v.dtype:
        raise ValueError("q, k and v must have one dtype")
    q4, k4, v4 = _heads4(q, "q"), _heads4(k, "k"), _heads4(v, "v")
    b, nq, hq, d = q4.shape
    kb, nk, hkv, kd = ks = k4.shape
    if v4.shape != ks or kd != d or kb != b:
        raise ValueError(f"shapes do not fit: q {tuple(q.shape)}, k {tuple(k.shape)}, v {tuple(v.shape)}")
    if hkv < 1 or hq < 1 or hq % hkv:
        raise ValueError(f"{hq} query heads cannot share {hkv} key heads evenly")
    nseq = 0
    if packed:
        if q_offsets is None or k_offsets is None or q_lens is not None or k_lens is not None:
            raise ValueError("packed sequences take q_offsets and k_offsets, and no lengths")
        nseq = q_offsets.numel() - 1
        if nseq < 1:
            raise ValueError("offsets need at least two entries")
        q_offsets, k_offsets = _int32(q_offsets, nseq + 1, "q_offsets"), _int32(k_offsets, nseq + 1, "k_offsets")
    if q_lens is not None:
        q_lens = _int32(q_lens, b, "q_lens")
    if k_lens is not None:
        k_lens = _int32(k_lens, b, "k_lens")
    _ATTENTION.pack_into(lane.memory, 0, _dtype(q, "q, k and v"), b, nq, nk, hq, hkv, d, 1 if causal else 0, window,
                         d ** -0.5 if scale is None else scale, nseq, 0, _address(q_lens), _address(k_lens), _address(q_offsets), _address(k_offsets))
    return q4, k4, v4, (hq, nq) if nseq else (b, hq, nq), (q_lens, k_lens, q_offsets, k_offsets)


def attention_forward(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, causal: bool = True, window: int = 0, scale: Optional[float] = None,
                      q_lens: Optional[torch.Tensor] = None, k_lens: Optional[torch.Tensor] = None,
                      q_offsets: Optional[torch.Tensor] = None, k_offsets: Optional[torch.Tensor] = None) -> Tuple[torch.Tensor, torch.Tensor]:
    """(o, lse).  q: [batch, tokens, heads, dim]; k, v: [batch, tokens, kv heads, dim], heads a multiple of kv heads; any strides with a
    contiguous last dimension.  q_lens, k_lens (int32 [batch]): how many tokens of each row count.  With q_offsets and k_offsets (int32
    [sequences + 1]) the tensors are [tokens, heads, dim] and hold packed sequences.  causal aligns the last query with the last key;
    window > 0 limits it to that many keys.  scale: dim ** -0.5 by default.  lse: fp32 [batch, heads, tokens] ([heads, tokens] packed)."""
    index = _on(q, k, v, q_lens, k_lens, q_offsets, k_offsets)
    if index != _current_device():
        with torch.cuda.device(index):
            return attention_forward(q, k, v, causal, window, scale, q_lens, k_lens, q_offsets, k_offsets)
    lane = _lane(index)
    q4, k4, v4, stat, keep = _attention_call(lane, q, k, v, causal, window, scale, q_lens, k_lens, q_offsets, k_offsets)
    o, lse = _like(q4), q.new_empty(stat, dtype=torch.float32)
    a, b, c, d, h = q4.stride(), k4.stride(), v4.stride(), o.stride(), lane.heads
    _HEADS[4].pack_into(lane.memory, _DESC_BYTES, q4.data_ptr(), a[0], a[1], a[2], k4.data_ptr(), b[0], b[1], b[2], v4.data_ptr(), c[0], c[1], c[2],
                        o.data_ptr(), d[0], d[1], d[2])
    rc = _attention_forward(lane.handle, lane.desc, h[0], h[1], h[2], h[3], lse.data_ptr(), _raw_stream(index))
    if rc:
        _refused(rc, "muon_attention_forward")
    return o if len(stat) == 3 else o[0], lse


def attention_backward(do: torch.Tensor, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, o: torch.Tensor, lse: torch.Tensor,
                       causal: bool = True, window: int = 0, scale: Optional[float] = None,
                       q_lens: Optional[torch.Tensor] = None, k_lens: Optional[torch.Tensor] = None,
                       q_offsets: Optional[torch.Tensor] = None, k_offsets: Optional[torch.Tensor] = None
                       ) -> Tuple[torch.Tensor, torch.Tensor, torch.Tensor]:
    """(dq, dk, dv) from what `attention_forward` took and gave."""
    index = _on(q, k, v, do, o, lse, q_lens, k_lens, q_offsets, k_offsets)
    if index != _current_device():
        with torch.cuda.device(index):
            return attention_backward(do, q, k, v, o, lse, causal, window, scale, q_lens, k_lens, q_offsets, k_offsets)
    lane = _lane(index)
    q4, k4, v4, stat, keep = _attention_call(lane, q, k, v, causal, window, scale, q_lens, k_lens, q_offsets, k_offsets)
    if do.shape != q.shape or o.shape != q.shape or do.dtype != q.dtype or o.dtype != q.dtype:
        raise ValueError("do and o must have the shape and dtype of q")
    if lse.shape != stat or lse.dtype != torch.float32:
        raise ValueError(f"lse must be fp32 of shape {tuple(stat)}")
    do4, o4, lse = _heads4(do, "do"), _heads4(o, "o"), lse.contiguous()
    dq, dk, dv = _like(q4), _like(k4), _like(v4)
    n = mb.muon_attention_workspace_bytes(lane.desc)
    ws = q.new_empty(n, dtype=torch.uint8) if n else None
    values = []
    for t in (do4, q4, k4, v4, o4, dq, dk, dv):
        s = t.stride()
        values += (t.data_ptr(), s[0], s[1], s[2])
    _HEADS[8].pack_into(lane.memory, _DESC_BYTES, *values)
    h = lane.heads
    rc = _attention_backward(lane.handle, lane.desc, h[0], h[1], h[2], h[3], h[4], lse.data_ptr(), h[5], h[6], h[7], _address(ws), n,
                             _raw_stream(index))
    if rc:
        _refused(rc, "muon_attention_backward")
    return (dq, dk, dv) if len(stat) == 3 else (dq[0], dk[0], dv[0])


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
