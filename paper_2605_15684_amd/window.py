"""Torch-facing binding of causal attention with a sliding window and sinks (include/ssba_window.h).

Argument marshalling only, like ssba.py: tensors are checked, outputs and scratch allocated with torch, and raw device
pointers plus the current HIP stream of the tensors' device passed to the HIP kernels in libssba.so.  Importing fails
if the library is not built.

    o, lse = window.forward(q, k, v, window=1024, sinks=4)              # q [B, H, T, D]; k, v [B, H_kv, T, D]
    dq, dk, dv = window.backward(q, k, v, o, do, lse, window=1024, sinks=4)

or with packed sequences: q [rows, H, D]; k, v [rows, H_kv, D]; cu int32 [sequences + 1] (where each begins).  The form
that reads the paged cache is cache.attend_window.
"""
from __future__ import annotations

import ctypes
import struct
from typing import Optional, Tuple

import torch

from . import _lib

_L = _lib.load()   # fail loudly at import if the HIP library is missing

__all__ = ["forward", "backward", "SsbaError"]

SsbaError = _lib.SsbaError
_DTYPES = {torch.bfloat16: _lib.DT_BF16, torch.float32: _lib.DT_F32}
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or \
    (lambda index: torch.cuda.current_stream(index).cuda_stream)
_current_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)


def _call(index: int, fn, name: str, *args) -> None:
    """fn(*args, stream) on the current stream of GPU `index`."""
    if _current_device() == index:
        st = fn(*args, _raw_stream(index))
    else:
        with torch.cuda.device(index):
            st = fn(*args, _raw_stream(index))
    if st:
        _lib.check(st, name)


# ssba_window and ssba_window_grads as bytes: a call of this module costs a few microseconds on the host, of which
# filling ctypes structures would be as many again.
_DESC = struct.Struct("=10if4xQ12q")
_GRADS = struct.Struct("=12q")
assert _DESC.size == ctypes.sizeof(_lib.WindowDesc) and _GRADS.size == ctypes.sizeof(_lib.WindowGrads)


def _contiguous(shape) -> Tuple[int, int, int]:
    """(batch, head, row) strides of a contiguous tensor."""
    if len(shape) == 3:
        _, h, d = shape
        return 0, d, h * d
    _, h, n, d = shape
    return h * n * d, n * d, d


def _strides(t, shape, dtype, index: int, what: str) -> Tuple[int, int, int]:
    """Checks a tensor of a shape, type and device; its (batch, head, row) strides."""
    if not isinstance(t, torch.Tensor) or t.dtype is not dtype or t.shape != shape:
        raise ValueError(f"{what}: expected a {dtype} GPU tensor of shape {tuple(shape)}")
    if t.get_device() != index:
        raise ValueError(f"{what}: all tensors must be on one device")
    if t.is_contiguous():
        return _contiguous(shape)
    if len(shape) == 3:
        n, h, d = shape
        st, sh, sc = t.stride()
        b, sb = 1, 0
    else:
        b, h, n, d = shape
        sb, sh, st, sc = t.stride()
    if sc != 1:
        raise ValueError(f"{what}: channel stride must be 1")
    # A dimension of one has no stride that matters; torch may report any.
    st = st if n > 1 else d
    sh = sh if h > 1 else d
    sb = sb if b > 1 else 0
    if st < d or sh < d or (b > 1 and sb < d):
        raise ValueError(f"{what}: rows and heads must not overlap")
    return sb, sh, st


def _place(t, like, dtype, index: int, what: str):
    """A tensor of the shape of `like` (None: allocated) and its strides."""
    if t is not None:
        return t, _strides(t, like.shape, dtype, index, what)
    return torch.empty_like(like, memory_format=torch.contiguous_format), _contiguous(like.shape)


def _desc(q, k, v, o, window: int, sinks: int, scale: Optional[float], cu, max_len: Optional[int]) -> bytes:
    """ssba_window of a call, its tensors checked; o None: a contiguous one that is still to be allocated."""
    if not isinstance(q, torch.Tensor) or not q.is_cuda or q.dim() not in (3, 4) or q.dtype not in _DTYPES:
        raise ValueError("q: expected a [B, H, T, D] or [rows, H, D] GPU tensor, bf16 or fp32")
    if not isinstance(k, torch.Tensor) or k.dim() != q.dim():
        raise ValueError("k: expected a tensor of q's dimensions")
    index, dtype, qs, kv = q.get_device(), q.dtype, q.shape, k.shape[1]
    if len(qs) == 4:
        if cu is not None:
            raise ValueError("cu goes with packed [rows, H, D] tensors")
        batch, heads, rows, d = qs
        shape, seqs, at = torch.Size((batch, kv, rows, d)), 0, 0
    else:
        rows, heads, d = qs
        batch, shape = 1, torch.Size((rows, kv, d))
        if not isinstance(cu, torch.Tensor) or cu.dtype is not torch.int32 or cu.dim() != 1 or cu.shape[0] < 2 or \
                not cu.is_contiguous() or cu.get_device() != index:
            raise ValueError("cu: expected a contiguous int32 tensor [sequences + 1] on q's device with packed tensors")
        seqs, at = cu.shape[0] - 1, cu.data_ptr()
    if kv < 1 or heads % kv:
        raise ValueError("q must have a multiple of k's heads")
    window, sinks, max_len = int(window), int(sinks), int(max_len or 0)
    if window < 1 or sinks < 0:
        raise ValueError("window must be 1 or more, sinks 0 or more")
    if scale is None:
        scale = 0.0
    else:
        scale = ctypes.c_float(scale).value
        if not scale > 0.0:
            raise ValueError("scale must be positive in fp32 (None: 1 / sqrt(D))")
    os = _contiguous(qs) if o is None else _strides(o, qs, dtype, index, "out")
    strides = _strides(q, qs, dtype, index, "q") + _strides(k, shape, dtype, index, "k") + \
        _strides(v, shape, dtype, index, "v") + os
    try:
        return _DESC.pack(batch, rows, heads, kv, d, _DTYPES[dtype], window, sinks, seqs, max_len, scale, at, *strides)
    except struct.error as e:
        raise ValueError(f"shape, window, sinks or max_len: outside int32 ({e})") from None


def _lse_shape(q):
    return (q.shape[1], q.shape[0]) if q.dim() == 3 else q.shape[:3]


def _check_lse(lse, q):
    if not (isinstance(lse, torch.Tensor) and lse.dtype is torch.float32 and lse.get_device() == q.get_device() and
            lse.is_contiguous() and lse.shape == _lse_shape(q)):
        raise ValueError(f"lse: expected a contiguous fp32 tensor of shape {tuple(_lse_shape(q))} on q's device")


def forward(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, *, window: int, sinks: int = 0,
            scale: Optional[float] = None, cu: Optional[torch.Tensor] = None, max_len: Optional[int] = None,
            out: Optional[torch.Tensor] = None, lse: Optional[torch.Tensor] = None) -> Tuple[torch.Tensor, torch.Tensor]:
    """Attention of every token over itself, the window - 1 tokens before it and the first `sinks` tokens of its
    sequence.  Returns (out, lse): lse fp32 [B, H, T], or [H, rows] of packed tensors, is what `backward` needs.
    scale: positive; None: 1 / sqrt(D).  max_len: about the longest packed sequence (work is split by it, results
    differ by the rounding of partial sums).  Rows of no sequence are left as they are."""
    desc = _desc(q, k, v, out, window, sinks, scale, cu, max_len)
    if out is None:
        out = torch.empty_like(q, memory_format=torch.contiguous_format)
    if lse is None:
        lse = q.new_empty(_lse_shape(q), dtype=torch.float32)
    else:
        _check_lse(lse, q)
    _call(q.get_device(), _L.ssba_window_forward, "ssba_window_forward", desc, q.data_ptr(), k.data_ptr(), v.data_ptr(),
          out.data_ptr(), lse.data_ptr())
    return out, lse


def backward(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, out: torch.Tensor, dout: torch.Tensor, lse: torch.Tensor,
             *, window: int, sinks: int = 0, scale: Optional[float] = None, cu: Optional[torch.Tensor] = None,
             max_len: Optional[int] = None, dq: Optional[torch.Tensor] = None, dk: Optional[torch.Tensor] = None,
             dv: Optional[torch.Tensor] = None,
             scratch: Optional[torch.Tensor] = None) -> Tuple[torch.Tensor, torch.Tensor, torch.Tensor]:
    """Gradients (dq, dk, dv) of `forward` for the upstream gradient `dout`, with its out, lse and arguments.  Rows of
    no sequence are left as they are."""
    if out is None:
        raise ValueError("out: expected the forward's")
    desc = _desc(q, k, v, out, window, sinks, scale, cu, max_len)
    _check_lse(lse, q)
    index, dtype = q.get_device(), q.dtype
    ds = _strides(dout, q.shape, dtype, index, "dout")
    dq, dqs = _place(dq, q, dtype, index, "dq")
    dk, dks = _place(dk, k, dtype, index, "dk")
    dv, dvs = _place(dv, k, dtype, index, "dv")
    grads = _GRADS.pack(*ds, *dqs, *dks, *dvs)
    size = ctypes.c_size_t(0)
    _lib.check(_L.ssba_window_backward_workspace_size(desc, size), "ssba_window_backward_workspace_size")
    if scratch is None:
        scratch = q.new_empty(size.value, dtype=torch.uint8)
    elif not (isinstance(scratch, torch.Tensor) and scratch.get_device() == index and scratch.is_contiguous()):
        raise ValueError("scratch must be a contiguous GPU tensor on q's device")
    _call(index, _L.ssba_window_backward, "ssba_window_backward", desc, grads, q.data_ptr(), k.data_ptr(),
          v.data_ptr(), out.data_ptr(), dout.data_ptr(), lse.data_ptr(), dq.data_ptr(), dk.data_ptr(), dv.data_ptr(),
          scratch.data_ptr(), scratch.numel() * scratch.element_size())
    return dq, dk, dv
