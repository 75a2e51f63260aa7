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


def _int32(what: str, *numbers) -> None:
    """The library's numbers are int32, and ctypes would cut larger ones."""
    for x in numbers:
        if not -0x80000000 <= x < 0x80000000:
            raise ValueError(f"{what}: outside int32")


def _strides(t, shape, like, what: str) -> _lib.Strides:
    """Checks a tensor of `shape` and of like's type and device; its strides."""
    if not (isinstance(t, torch.Tensor) and t.is_cuda and t.dtype == like.dtype and t.shape == shape):
        raise ValueError(f"{what}: expected a {like.dtype} GPU tensor of shape {tuple(shape)}")
    if t.get_device() != like.get_device():
        raise ValueError(f"{what}: all tensors must be on one device")
    if t.dim() == 3:
        (n, h, d), (st, sh, sc) = t.shape, t.stride()
        b, sb = 1, 0
    else:
        (b, h, n, d), (sb, sh, st, sc) = t.shape, t.stride()
    if t.numel() == 0:
        return _lib.Strides(0, 0, 0)
    if sc != 1:
        raise ValueError(f"{what}: channel stride must be 1")
    # A dimension of one has no stride that matters; torch may report any.
    st = st if n > 1 else d
    sh = sh if h > 1 else d
    sb = sb if b > 1 else 0
    if st < d or sh < d or (b > 1 and sb < d):
        raise ValueError(f"{what}: rows and heads must not overlap")
    return _lib.Strides(sb, sh, st)


def _desc(q, k, v, o, window: int, sinks: int, scale: Optional[float], cu, max_len: Optional[int]):
    if not (isinstance(q, torch.Tensor) and q.is_cuda and q.dim() in (3, 4) and q.dtype in _DTYPES):
        raise ValueError("q: expected a [B, H, T, D] or [rows, H, D] GPU tensor, bf16 or fp32")
    if not (isinstance(k, torch.Tensor) and k.dim() == q.dim()):
        raise ValueError("k: expected a tensor of q's dimensions")
    if q.dim() == 4:
        if cu is not None:
            raise ValueError("cu goes with packed [rows, H, D] tensors")
        batch, heads, rows, d = q.shape
        kv = k.shape[1]
        shape, seqs, at = (batch, kv, rows, d), 0, None
    else:
        rows, heads, d = q.shape
        kv = k.shape[1]
        batch, shape = 1, (rows, kv, d)
        if not (isinstance(cu, torch.Tensor) and cu.dtype is torch.int32 and cu.dim() == 1 and cu.shape[0] > 1 and
                cu.is_contiguous() and cu.get_device() == q.get_device()):
            raise ValueError("cu: expected a contiguous int32 tensor [sequences + 1] on q's device with packed tensors")
        seqs, at = cu.shape[0] - 1, cu.data_ptr()
    if kv < 1 or heads % kv:
        raise ValueError("q must have a multiple of k's heads")
    window, sinks, max_len = int(window), int(sinks), int(max_len or 0)
    _int32("shape, window, sinks or max_len", batch, rows, heads, window, sinks, max_len, seqs)
    if window < 1 or sinks < 0:
        raise ValueError("window must be 1 or more, sinks 0 or more")
    if scale is None:
        scale = 0.0
    else:
        scale = ctypes.c_float(scale).value
        if not scale > 0.0:
            raise ValueError("scale must be positive in fp32 (None: 1 / sqrt(D))")
    return _lib.WindowDesc(batch, rows, heads, kv, d, _DTYPES[q.dtype], window, sinks, seqs, max_len, scale, at,
                           _strides(q, q.shape, q, "q"), _strides(k, shape, q, "k"), _strides(v, shape, q, "v"),
                           _strides(o, q.shape, q, "out"))


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
    scale: positive; None: 1 / sqrt(D).  max_len: about the longest packed sequence (work is split by it; results are
    not).  Rows of no sequence are left as they are."""
    if out is None and isinstance(q, torch.Tensor):
        out = torch.empty_like(q, memory_format=torch.contiguous_format)
    desc = _desc(q, k, v, out, window, sinks, scale, cu, max_len)
    if lse is None:
        lse = torch.empty(_lse_shape(q), dtype=torch.float32, device=q.device)
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
    desc = _desc(q, k, v, out, window, sinks, scale, cu, max_len)
    _check_lse(lse, q)
    mk = lambda t, like: torch.empty_like(like, memory_format=torch.contiguous_format) if t is None else t
    dq, dk, dv = mk(dq, q), mk(dk, k), mk(dv, v)
    grads = _lib.WindowGrads(_strides(dout, q.shape, q, "dout"), _strides(dq, q.shape, q, "dq"),
                             _strides(dk, k.shape, q, "dk"), _strides(dv, v.shape, q, "dv"))
    size = ctypes.c_size_t(0)
    _lib.check(_L.ssba_window_backward_workspace_size(desc, size), "ssba_window_backward_workspace_size")
    if scratch is None:
        scratch = torch.empty(size.value, dtype=torch.uint8, device=q.device)
    elif not (isinstance(scratch, torch.Tensor) and scratch.get_device() == q.get_device() and scratch.is_contiguous()):
        raise ValueError("scratch must be a contiguous GPU tensor on q's device")
    _call(q.get_device(), _L.ssba_window_backward, "ssba_window_backward", desc, grads, q.data_ptr(), k.data_ptr(),
          v.data_ptr(), out.data_ptr(), dout.data_ptr(), lse.data_ptr(), dq.data_ptr(), dk.data_ptr(), dv.data_ptr(),
          scratch.data_ptr(), scratch.numel() * scratch.element_size())
    return dq, dk, dv
