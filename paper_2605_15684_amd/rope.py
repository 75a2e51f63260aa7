"""Torch-facing binding of the rotary positions with several axes (include/ssba_rope.h).

Argument marshalling only, like ssba.py: tensors are checked, outputs allocated with torch, and raw device pointers
plus the current HIP stream of the tensors' device passed to the HIP kernel in libssba.so.  Importing fails if the
library is not built.

    turn = rope.plan(128, (16, 24, 24), theta=10000.0)      # pairs that go by (time, height, width): once
    q, k = rope.rotate(turn, pos, q, k)                     # pos int32 [tokens, 3]; q [tokens, heads, D]
    ...
    dq, dk = rope.rotate(turn, pos, dq, dk, inverse=True)   # gradients, turned back
"""
from __future__ import annotations

import ctypes
import math
import struct
from typing import Optional, Sequence

import torch

from . import _lib

_L = _lib.load()   # fail loudly at import if the HIP library is missing

__all__ = ["Plan", "plan", "rotate", "SsbaError"]

SsbaError = _lib.SsbaError
_DTYPES = {torch.bfloat16: _lib.DT_BF16, torch.float32: _lib.DT_F32}
_PAIRS = {"adjacent": 0, "halves": 1}
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or \
    (lambda index: torch.cuda.current_stream(index).cuda_stream)
_current_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)


class Plan:
    """How the pairs of a head turn: `axis` (which position a pair goes by, -1: it stays) and `freq` (radians a
    position) of each of the head_dim / 2 pairs; `pairs` "adjacent": channels (2j, 2j+1), "halves": (j, j + D/2).
    Holds host tables only, so it serves any device and stream."""

    __slots__ = ("head_dim", "axes", "pairs", "desc", "_axis", "_freq")

    def __init__(self, head_dim: int, axes: int, axis: Sequence[int], freq: Sequence[float], pairs: str = "adjacent"):
        if head_dim not in (64, 128):
            raise ValueError("head_dim must be 64 or 128")
        if not 1 <= axes <= 4:
            raise ValueError("axes must be 1 .. 4")
        if pairs not in _PAIRS:
            raise ValueError("pairs must be 'adjacent' or 'halves'")
        half = head_dim // 2
        axis, freq = [int(a) for a in axis], [float(f) for f in freq]
        if len(axis) != half or len(freq) != half:
            raise ValueError(f"axis and freq: expected {half} values")
        if any(not -1 <= a < axes for a in axis):
            raise ValueError("axis: outside -1 .. axes-1")
        if any(not abs(f) <= 2.0 ** 20 for f in freq):
            raise ValueError("freq: must be finite and at most 2^20")
        self.head_dim, self.axes, self.pairs = head_dim, axes, pairs
        self._axis, self._freq = (ctypes.c_int32 * half)(*axis), (ctypes.c_double * half)(*freq)
        self.desc = _lib.RopeDesc(head_dim, _PAIRS[pairs], axes, ctypes.addressof(self._axis),
                                  ctypes.addressof(self._freq))


def plan(head_dim: int, sections: Sequence[int], *, theta: float = 10000.0, spectrum: str = "axis",
         pairs: str = "adjacent", step: Optional[Sequence[float]] = None) -> Plan:
    """The first sections[0] pairs go by axis 0, the next sections[1] by axis 1 and so on; further pairs stay.
    spectrum "axis": pair i of a section of n has frequency theta^(-i/n); "shared": pair j of all D/2 has
    theta^(-j/(D/2)).  step: what one position of each axis counts for (1.0; a video of half the frame rate: 2.0 for
    its time)."""
    half = head_dim // 2
    sections = [int(n) for n in sections]
    if any(n < 0 for n in sections) or sum(sections) > half:
        raise ValueError(f"sections: expected sizes of at most {half} pairs together")
    if spectrum not in ("axis", "shared"):
        raise ValueError("spectrum must be 'axis' or 'shared'")
    if not (theta > 0 and math.isfinite(theta)):
        raise ValueError("theta must be positive")
    step = [1.0] * len(sections) if step is None else [float(x) for x in step]
    if len(step) != len(sections):
        raise ValueError("step: expected one value an axis")
    axis, freq = [-1] * half, [0.0] * half
    j = 0
    for a, n in enumerate(sections):
        for i in range(n):
            axis[j], freq[j] = a, step[a] * theta ** -(i / n if spectrum == "axis" else j / half)
            j += 1
    return Plan(head_dim, len(sections), axis, freq, pairs)


# ssba_rope_tensor as bytes: a call of this module costs a few microseconds on the host, of which filling ctypes
# structures would be as many again.
_TENSOR = struct.Struct("=i4xQQ6q")
assert _TENSOR.size == ctypes.sizeof(_lib.RopeTensor)


def _tensor(t, dtype, dim: int, batch: int, rows: int, d: int, index: int, what: str):
    """Checks a [tokens, heads, D] or [B, H, T, D] tensor; its heads and (batch, head, token) strides."""
    if not isinstance(t, torch.Tensor) or t.dtype is not dtype or t.dim() != dim:
        raise ValueError(f"{what}: expected a tensor of q's type and dimensions")
    if t.get_device() != index:
        raise ValueError(f"{what}: all tensors must be on one device")
    if dim == 3:
        n, h, e = t.shape
        b = 1
    else:
        b, h, n, e = t.shape
    if e != d or b != batch or n != rows:
        raise ValueError(f"{what}: expected the tokens of q, and head_dim {d} as the plan")
    if t.is_contiguous():
        return (h, 0, d, h * d) if dim == 3 else (h, h * n * d, n * d, d)
    if dim == 3:
        st, sh, sc = t.stride()
        sb = 0
    else:
        sb, sh, st, sc = t.stride()
    if sc != 1:
        raise ValueError(f"{what}: channel stride must be 1")
    # A dimension of one has no stride that matters; torch may report any.
    st = st if n > 1 else d
    sh = sh if h > 1 else d
    sb = sb if b > 1 else 0
    if st < d or sh < d or (b > 1 and sb < d):
        raise ValueError(f"{what}: rows and heads must not overlap")
    return h, sb, sh, st


def _pair(t, out, dtype, dim: int, batch: int, rows: int, d: int, index: int, what: str):
    """A tensor and where it goes (None: allocated): (heads, output, ssba_rope_tensor)."""
    h, *strides = _tensor(t, dtype, dim, batch, rows, d, index, what)
    if out is None:
        out = torch.empty_like(t, memory_format=torch.contiguous_format)
        to = (0, d, h * d) if dim == 3 else (h * rows * d, rows * d, d)
    else:
        if isinstance(out, torch.Tensor) and out.shape != t.shape:
            raise ValueError(f"{what}_out: expected the shape of {what}")
        to = _tensor(out, dtype, dim, batch, rows, d, index, what + "_out")[1:]
    return h, out, _TENSOR.pack(h, t.data_ptr(), out.data_ptr(), *strides, *to)


def rotate(plan: Plan, pos: torch.Tensor, q: torch.Tensor, k: Optional[torch.Tensor] = None, *, inverse: bool = False,
           q_out: Optional[torch.Tensor] = None, k_out: Optional[torch.Tensor] = None):
    """q (and k, of another number of heads) turned by the positions of their tokens; with `inverse` turned back, which
    is the gradient.  q [tokens, heads, D] with pos int32 [tokens, axes], or [B, H, T, D] with pos [T, axes] or
    [B, T, axes].  q_out and k_out may be q and k themselves.  Returns q_out or (q_out, k_out)."""
    if not isinstance(plan, Plan):
        raise ValueError("plan: expected a rope.Plan")
    if not isinstance(q, torch.Tensor) or not q.is_cuda or q.dim() not in (3, 4) or q.dtype not in _DTYPES:
        raise ValueError("q: expected a [tokens, heads, D] or [B, H, T, D] GPU tensor, bf16 or fp32")
    index, dim, dtype, d, shape = q.get_device(), q.dim(), q.dtype, plan.head_dim, q.shape
    batch, rows = (1, shape[0]) if dim == 3 else (shape[0], shape[2])
    own = False   # positions of each batch entry
    if isinstance(pos, torch.Tensor) and pos.dtype is torch.int32 and pos.get_device() == index:
        where = tuple(pos.shape)
        own = where == (batch, rows, plan.axes) and dim == 4
        fits = own or where == (rows, plan.axes)
    else:
        fits = False
    if not fits:
        raise ValueError(f"pos: expected an int32 tensor [tokens, {plan.axes}]" +
                         (f" or [B, T, {plan.axes}]" if dim == 4 else "") + " on q's device")
    step = pos.stride()
    if plan.axes > 1 and step[-1] != 1 and pos.numel():
        raise ValueError("pos: the axes of a token must be contiguous")
    most, q_out, desc = _pair(q, q_out, dtype, dim, batch, rows, d, index, "q")
    if k is not None:
        h, k_out, more = _pair(k, k_out, dtype, dim, batch, rows, d, index, "k")
        most = max(most, h)
        desc += more
    elif k_out is not None:
        raise ValueError("k_out without k")
    if batch >= 1 << 31 or rows >= 1 << 31 or most >= 1 << 31:
        raise ValueError("q: outside int32")
    if q.numel() or (k is not None and k.numel()):
        args = (plan.desc, _DTYPES[dtype], 1 if inverse else 0, batch, rows, pos.data_ptr(),
                step[0] if own and batch > 1 else 0, step[-2] if rows > 1 else 0,
                1 if k is None else 2, desc)
        if _current_device() == index:
            status = _L.ssba_rope_rotate(*args, _raw_stream(index))
        else:
            with torch.cuda.device(index):
                status = _L.ssba_rope_rotate(*args, _raw_stream(index))
        if status:
            _lib.check(status, "ssba_rope_rotate")
    return q_out if k is None else (q_out, k_out)
