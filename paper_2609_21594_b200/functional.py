"""torch front end of the layer operators: layer norm, rotary positions and attention, forward and backward.

What a training program needs around the matrices that `optim.Muon` updates.  Argument checks and marshalling only: the arithmetic runs
in the CUDA library, on the current stream of the tensors' device.  `layer_norm`, `rotary` and `attention` are differentiable;
the `*_forward` / `*_backward` pairs are the same calls for programs that keep their own tape.  Each host thread has a context
of its own per device (autograd calls backward passes from another thread).
"""
from __future__ import annotations

import ctypes as C
import threading
from typing import Optional, Sequence, Tuple

import numpy as np
import torch

from . import binding as mb
from .binding import muon_rotary_frequencies as rotary_frequencies  # noqa: F401  (part of this module's interface)

_DTYPES = {torch.bfloat16: mb.DTYPE_BF16, torch.float32: mb.DTYPE_FP32}
_local = threading.local()


def context(device: Optional[torch.device] = None) -> mb.Context:
    """This thread's context of a device (default: the current one): the one the functions of this module use there."""
    index = torch.cuda.current_device() if device is None or device.index is None else device.index
    per = getattr(_local, "contexts", None)
    if per is None:
        per = _local.contexts = {}
    ctx = per.get(index)
    if ctx is None:
        with torch.cuda.device(index):
            ctx = per[index] = mb.Context()
    return ctx


def _dtype(t: torch.Tensor, what: str) -> int:
    d = _DTYPES.get(t.dtype)
    if d is None:
        raise ValueError(f"{what} must be bf16 or fp32, not {t.dtype}")
    return d


def _on(t: torch.Tensor, *others: Optional[torch.Tensor]) -> None:
    if not t.is_cuda:
        raise ValueError("the layer operators take CUDA tensors (there is no CPU fallback)")
    for o in others:
        if o is not None and o.device != t.device:
            raise ValueError(f"tensors on {o.device} and {t.device} in one call")


class _Guard:
    """Makes the tensors' device current for the call when it is not."""

    def __init__(self, t: torch.Tensor):
        self._guard = None if t.device.index == torch.cuda.current_device() else torch.cuda.device(t.device)

    def __enter__(self):
        if self._guard is not None:
            self._guard.__enter__()

    def __exit__(self, *exc):
        if self._guard is not None:
            self._guard.__exit__(*exc)


def _ptr(t: Optional[torch.Tensor]) -> Optional[int]:
    return None if t is None else t.data_ptr()


# ------------------------------------------------------------------------------------------------ layer norm
def _rows(t: torch.Tensor, what: str) -> torch.Tensor:
    """[..., cols] as [rows, cols] with contiguous rows: a view where the strides allow one, else a copy."""
    if t.dim() < 1 or t.shape[-1] < 1:
        raise ValueError(f"{what} needs a last dimension of at least one element")
    r = t.reshape(-1, t.shape[-1])
    return r if (r.shape[1] == 1 or r.stride(1) == 1) and (r.shape[0] <= 1 or r.stride(0) >= r.shape[1]) else r.contiguous()


def _ld(r: torch.Tensor) -> int:
    return max(r.stride(0), r.shape[1]) if r.shape[0] > 1 else r.shape[1]


def _param(p: Optional[torch.Tensor], cols: int, what: str) -> Optional[torch.Tensor]:
    if p is None:
        return None
    if p.shape != (cols,):
        raise ValueError(f"{what} must have shape ({cols},), not {tuple(p.shape)}")
    return p.contiguous()


def _norm_desc(x: torch.Tensor, r: torch.Tensor, weight, bias, eps: float, center: bool) -> mb.NormDesc:
    if weight is not None and bias is not None and weight.dtype != bias.dtype:
        raise ValueError("weight and bias must have one dtype")
    p = weight if weight is not None else bias
    return mb.NormDesc(_dtype(x, "x"), mb.DTYPE_FP32 if p is None else _dtype(p, "weight and bias"), 1 if center else 0, r.shape[1], r.shape[0],
                       eps, 0)


def layer_norm_forward(x: torch.Tensor, weight: Optional[torch.Tensor] = None, bias: Optional[torch.Tensor] = None, eps: float = 1e-5,
                       center: bool = True) -> Tuple[torch.Tensor, Optional[torch.Tensor], torch.Tensor]:
    """(y, mean, rstd) over the last dimension; center=False is RMS norm and gives mean = None.  mean, rstd: fp32, x.shape[:-1]."""
    _on(x, weight, bias)
    r = _rows(x, "x")
    weight, bias = _param(weight, r.shape[1], "weight"), _param(bias, r.shape[1], "bias")
    desc = _norm_desc(x, r, weight, bias, eps, center)
    with _Guard(x):
        y = torch.empty(x.shape, dtype=x.dtype, device=x.device)
        mean = torch.empty(x.shape[:-1], dtype=torch.float32, device=x.device) if center else None
        rstd = torch.empty(x.shape[:-1], dtype=torch.float32, device=x.device)
        context(x.device).muon_layer_norm_forward(desc, r.data_ptr(), _ld(r), _ptr(weight), _ptr(bias), y.data_ptr(), r.shape[1], _ptr(mean),
                                                  rstd.data_ptr())
    return y, mean, rstd


def layer_norm_backward(dy: torch.Tensor, x: torch.Tensor, weight: Optional[torch.Tensor], mean: Optional[torch.Tensor], rstd: torch.Tensor,
                        bias: bool = True, bias_dtype: Optional[torch.dtype] = None
                        ) -> Tuple[torch.Tensor, Optional[torch.Tensor], Optional[torch.Tensor]]:
    """(dx, dweight, dbias); dweight is None without a weight, dbias unless `bias`.  The gradients have the weight's dtype (without a
    weight: bias_dtype, fp32 by default)."""
    _on(x, dy, weight, mean, rstd)
    if dy.shape != x.shape or dy.dtype != x.dtype:
        raise ValueError("dy must have the shape and dtype of x")
    if rstd.shape != x.shape[:-1] or (mean is not None and mean.shape != rstd.shape):
        raise ValueError("mean and rstd must have the shape of x without its last dimension")
    if rstd.dtype != torch.float32 or (mean is not None and mean.dtype != torch.float32):
        raise ValueError("mean and rstd must be fp32")
    r, g = _rows(x, "x"), _rows(dy, "dy")
    weight = _param(weight, r.shape[1], "weight")
    mean, rstd = None if mean is None else mean.contiguous(), rstd.contiguous()
    desc = _norm_desc(x, r, weight, None, 0.0, mean is not None)
    pt = weight.dtype if weight is not None else (bias_dtype or torch.float32)
    if pt not in _DTYPES:
        raise ValueError(f"gradients must be bf16 or fp32, not {pt}")
    desc.param_dtype = _DTYPES[pt]
    with _Guard(x):
        dx = torch.empty(x.shape, dtype=x.dtype, device=x.device)
        dw = torch.empty(r.shape[1], dtype=pt, device=x.device) if weight is not None else None
        db = torch.empty(r.shape[1], dtype=pt, device=x.device) if bias else None
        n = mb.muon_layer_norm_workspace_bytes(desc) if dw is not None or db is not None else 0
        ws = torch.empty(n, dtype=torch.uint8, device=x.device) if n else None
        context(x.device).muon_layer_norm_backward(desc, g.data_ptr(), _ld(g), r.data_ptr(), _ld(r), _ptr(weight), _ptr(mean), rstd.data_ptr(),
                                                   dx.data_ptr(), r.shape[1], _ptr(dw), _ptr(db), _ptr(ws), n)
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
    if t.dim() != 4:
        raise ValueError(f"{what} must be [batch, tokens, heads, dim] or [tokens, heads, dim]")
    return t if t.stride(3) == 1 or t.shape[3] == 1 else t.contiguous()


def _heads(t: torch.Tensor) -> mb.Heads:
    s = t.stride()
    return mb.Heads(t.data_ptr(), s[0], s[1], s[2])


def _like(t: torch.Tensor) -> torch.Tensor:
    return torch.empty(t.shape, dtype=t.dtype, device=t.device)


# ------------------------------------------------------------------------------------------------ rotary positions
def rotary_forward(tensors: Sequence[torch.Tensor], inv_freq, layout: str = "half", amplitude: float = 1.0,
                   positions: Optional[torch.Tensor] = None, offset: int = 0, inverse: bool = False,
                   out: Optional[Sequence[torch.Tensor]] = None) -> Tuple[torch.Tensor, ...]:
    """Turns up to four [batch, tokens, heads, dim] (or [tokens, heads, dim]) tensors that share positions, in one launch.

    inv_freq: host, fp64 radians per position of each pair (see `rotary_frequencies`); twice its length is the part of the head that is
    turned, the rest is copied.  layout: "half" (i with i + n/2) or "interleaved" (2i with 2i + 1).  positions: int32 [batch, tokens] on
    the device, else offset + 0, 1, 2...; offset is added to given positions too.  inverse turns back, which is the backward pass.
    out: tensors to write, which may be the inputs themselves."""
    tensors = list(tensors)
    if not 1 <= len(tensors) <= 4:
        raise ValueError("one to four tensors")
    if layout not in ("half", "interleaved"):
        raise ValueError("layout is 'half' or 'interleaved'")
    first = tensors[0]
    _on(first, positions, *tensors[1:])
    freq = np.ascontiguousarray(inv_freq, dtype=np.float64)
    xs = [_heads4(t, "a tensor") for t in tensors]
    b, n, _, d = xs[0].shape
    for t in xs[1:]:
        if t.shape[:2] != (b, n) or t.shape[3] != d or t.dtype != first.dtype:
            raise ValueError("the tensors must agree in batch, tokens, head size and dtype")
    if freq.ndim != 1 or not 1 <= freq.size <= d // 2:
        raise ValueError(f"inv_freq must hold one to {d // 2} frequencies for heads of {d}")
    if positions is not None:
        if positions.dtype != torch.int32 or positions.numel() != b * n:
            raise ValueError("positions must be int32, one for each token")
        positions = positions.contiguous()
    with _Guard(first):
        if out is None:
            res = [_like(t) for t in tensors]
        else:
            res = list(out)
            if len(res) != len(tensors) or any(o.shape != t.shape or o.dtype != t.dtype or o.device != t.device for o, t in zip(res, tensors)):
                raise ValueError("out must match the tensors")
            if any(o.stride(-1) != 1 and o.shape[-1] > 1 for o in res):
                raise ValueError("out must have a contiguous last dimension")
        items = (mb.RotaryItem * len(xs))()
        for i, (x, o) in enumerate(zip(xs, res)):
            items[i].inp, items[i].out, items[i].heads = _heads(x), _heads(o if o.dim() == 4 else o[None]), x.shape[2]
        desc = mb.RotaryDesc(_dtype(first, "the tensors"), 1 if layout == "interleaved" else 0, 1 if inverse else 0, d, 2 * freq.size, b, n,
                             amplitude, freq.ctypes.data, _ptr(positions), offset)
        context(first.device).muon_rotary(desc, items, len(xs))
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
def _int32(t: Optional[torch.Tensor], n: Optional[int], what: str) -> Optional[torch.Tensor]:
    if t is None:
        return None
    if t.dtype != torch.int32 or t.dim() != 1 or (n is not None and t.numel() != n):
        raise ValueError(f"{what} must be a 1-D int32 tensor" + ("" if n is None else f" of {n}"))
    return t.contiguous()


def _attention_call(q, k, v, causal, window, scale, q_lens, k_lens, q_offsets, k_offsets):
    """(descriptor, 4-D q, k, v, tensors the descriptor points into)"""
    _on(q, k, v, q_lens, k_lens, q_offsets, k_offsets)
    packed = q_offsets is not None or k_offsets is not None
    if q.dim() != (3 if packed else 4) or k.dim() != q.dim() or v.dim() != q.dim():
        raise ValueError("q, k, v are [batch, tokens, heads, dim], or [tokens, heads, dim] with offsets")
    if not (q.dtype == k.dtype == v.dtype):
        raise ValueError("q, k and v must have one dtype")
    if k.shape != v.shape or k.shape[-1] != q.shape[-1] or (not packed and k.shape[0] != q.shape[0]):
        raise ValueError(f"shapes do not fit: q {tuple(q.shape)}, k {tuple(k.shape)}, v {tuple(v.shape)}")
    q4, k4, v4 = _heads4(q, "q"), _heads4(k, "k"), _heads4(v, "v")
    b, nq, hq, d = q4.shape
    nk, hkv = k4.shape[1:3]
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
    q_lens, k_lens = _int32(q_lens, b, "q_lens"), _int32(k_lens, b, "k_lens")
    desc = mb.AttentionDesc(_dtype(q, "q, k and v"), b, nq, nk, hq, hkv, d, 1 if causal else 0, window, d ** -0.5 if scale is None else scale,
                            nseq, 0, _ptr(q_lens), _ptr(k_lens), _ptr(q_offsets), _ptr(k_offsets))
    return desc, q4, k4, v4, (q_lens, k_lens, q_offsets, k_offsets)


def attention_forward(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, causal: bool = True, window: int = 0, scale: Optional[float] = None,
                      q_lens: Optional[torch.Tensor] = None, k_lens: Optional[torch.Tensor] = None,
                      q_offsets: Optional[torch.Tensor] = None, k_offsets: Optional[torch.Tensor] = None) -> Tuple[torch.Tensor, torch.Tensor]:
    """(o, lse).  q: [batch, tokens, heads, dim]; k, v: [batch, tokens, kv heads, dim], heads a multiple of kv heads; any strides with a
    contiguous last dimension.  q_lens, k_lens (int32 [batch]): how many tokens of each row count.  With q_offsets and k_offsets (int32
    [sequences + 1]) the tensors are [tokens, heads, dim] and hold packed sequences.  causal aligns the last query with the last key;
    window > 0 limits it to that many keys.  scale: dim ** -0.5 by default.  lse: fp32 [batch, heads, tokens] ([heads, tokens] packed)."""
    desc, q4, k4, v4, keep = _attention_call(q, k, v, causal, window, scale, q_lens, k_lens, q_offsets, k_offsets)
    with _Guard(q):
        o = _like(q)
        lse = torch.empty((desc.q_heads, desc.q_tokens) if desc.num_seqs else (desc.batch, desc.q_heads, desc.q_tokens), dtype=torch.float32,
                          device=q.device)
        context(q.device).muon_attention_forward(desc, _heads(q4), _heads(k4), _heads(v4), _heads(o if o.dim() == 4 else o[None]), lse.data_ptr())
    return o, lse


def attention_backward(do: torch.Tensor, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, o: torch.Tensor, lse: torch.Tensor,
                       causal: bool = True, window: int = 0, scale: Optional[float] = None,
                       q_lens: Optional[torch.Tensor] = None, k_lens: Optional[torch.Tensor] = None,
                       q_offsets: Optional[torch.Tensor] = None, k_offsets: Optional[torch.Tensor] = None
                       ) -> Tuple[torch.Tensor, torch.Tensor, torch.Tensor]:
    """(dq, dk, dv) from what `attention_forward` took and gave."""
    desc, q4, k4, v4, keep = _attention_call(q, k, v, causal, window, scale, q_lens, k_lens, q_offsets, k_offsets)
    _on(q, do, o, lse)
    if do.shape != q.shape or o.shape != q.shape or do.dtype != q.dtype or o.dtype != q.dtype:
        raise ValueError("do and o must have the shape and dtype of q")
    want = (desc.q_heads, desc.q_tokens) if desc.num_seqs else (desc.batch, desc.q_heads, desc.q_tokens)
    if lse.shape != want or lse.dtype != torch.float32:
        raise ValueError(f"lse must be fp32 of shape {want}")
    do4, o4, lse = _heads4(do, "do"), _heads4(o, "o"), lse.contiguous()
    with _Guard(q):
        dq, dk, dv = _like(q), _like(k), _like(v)
        n = mb.muon_attention_workspace_bytes(desc)
        ws = torch.empty(n, dtype=torch.uint8, device=q.device) if n else None
        up = (lambda t: t[None]) if desc.num_seqs else (lambda t: t)
        context(q.device).muon_attention_backward(desc, _heads(do4), _heads(q4), _heads(k4), _heads(v4), _heads(o4), lse.data_ptr(),
                                                  _heads(up(dq)), _heads(up(dk)), _heads(up(dv)), _ptr(ws), n)
    return dq, dk, dv


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
