"""Python binding of the rotary positions (include/qwam.h): queries and keys turned by their tokens' positions on one or
several axes, in front of the paged cache and its attention (block.py).  As in `qwam`, arguments are checked here, every
step runs in the library's HIP kernel, and there is no fallback.

rope is differentiable in x: with an x that requires a gradient it records the inverse turn.  Positions and frequencies
have no gradient, and are refused where they require one.
"""

from __future__ import annotations

import ctypes
from dataclasses import dataclass
from typing import Optional, Sequence

import torch

from . import qwam as _q

X_TYPES = (torch.bfloat16, torch.float32)
POS_TYPES = (torch.int32, torch.float32)


@dataclass
class RopePlan:
    """The pairs of a head's channels that turn: pair i (channels 2i and 2i + 1 if interleaved, else i and i + pairs) by the
    position on axis[i] times inv_freq[i].  inv_freq: float32 [pairs], axis: int32 [pairs], on the GPU; a pair whose axis
    is none of the positions' does not turn, nor do channels from 2 * pairs on."""
    inv_freq: torch.Tensor
    axis: torch.Tensor
    interleaved: bool = False


def rope_plan(dims: Sequence[int], theta: float = 10000.0, interleaved: bool = False, device="cuda") -> RopePlan:
    """A plan that gives each axis a block of dims[a] channels' pairs, in order, with frequencies theta ** (-2 i / dims[a]),
    i = 0 .. dims[a] / 2 - 1."""
    dims = list(dims)
    if not dims or any(not isinstance(d, int) or d <= 0 or d % 2 for d in dims):
        raise ValueError(f"dims must be positive even integers, one for each axis (got {dims})")
    if not theta > 0:
        raise ValueError(f"theta must be positive (got {theta})")
    f = [theta ** (-2 * i / d) for d in dims for i in range(d // 2)]
    axis = [a for a, d in enumerate(dims) for _ in range(d // 2)]
    return RopePlan(torch.tensor(f, dtype=torch.float32, device=device), torch.tensor(axis, dtype=torch.int32, device=device),
                    bool(interleaved))


def _heads(t: torch.Tensor, name: str, dtype, shape) -> int:
    """Pointer of a [tokens][heads][dim] whose tokens may be apart (a slice of a layer's wider output)."""
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch.Tensor")
    if t.device.type != "cuda":
        raise ValueError(f"{name} must be a GPU tensor (got {t.device})")
    if t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype} (got {t.dtype})")
    if tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name} must have shape {tuple(shape)} (got {tuple(t.shape)})")
    if (t.shape[2] > 1 and t.stride(2) != 1) or (t.shape[1] > 1 and t.stride(1) != t.shape[2]):
        raise ValueError(f"{name} must be contiguous along its heads")
    return t.data_ptr()


def _rope(x, positions, plan, inverse, out, stream):
    if not isinstance(plan, RopePlan):
        raise TypeError("plan must be a RopePlan")
    if not isinstance(x, torch.Tensor) or x.dim() != 3:
        raise ValueError("x must be a tensor of three dimensions (tokens, heads, dim)")
    if x.dtype not in X_TYPES:
        raise TypeError(f"x must be {X_TYPES[0]} or {X_TYPES[1]} (got {x.dtype})")
    if not isinstance(positions, torch.Tensor) or positions.dim() != 2:
        raise ValueError("positions must be a tensor of two dimensions (tokens, axes)")
    if positions.dtype not in POS_TYPES:
        raise TypeError(f"positions must be {POS_TYPES[0]} or {POS_TYPES[1]} (got {positions.dtype})")
    if not isinstance(plan.inv_freq, torch.Tensor) or plan.inv_freq.dim() != 1:
        raise ValueError("plan.inv_freq must be a tensor of one dimension (pairs)")
    T, H, D = x.shape
    c = _q.QwamRopePlanC()
    c.heads, c.dim, c.pairs, c.interleaved = H, D, plan.inv_freq.shape[0], bool(plan.interleaved)
    c.positions, c.axes = positions.shape
    c.pos_f32, c.x_f32 = positions.dtype == torch.float32, x.dtype == torch.float32
    c.pos = _q._req(positions, "positions", positions.dtype, tuple(positions.shape))
    c.inv_freq = _q._req(plan.inv_freq, "plan.inv_freq", torch.float32, (c.pairs,))
    c.axis = _q._req(plan.axis, "plan.axis", torch.int32, (c.pairs,))
    px = _heads(x, "x", x.dtype, x.shape)
    _q._on_current_device("rope", stream, x=x, positions=positions, out=out, **{"plan.inv_freq": plan.inv_freq, "plan.axis": plan.axis})
    y = _q._empty(x.shape, x.dtype, x.device, stream) if out is None else out
    py = _heads(y, "out", x.dtype, x.shape)
    xs, ys = (t.stride(0) if T > 1 else 0 for t in (x, y))
    if out is not None and (px != py or xs != ys):
        # (memory between the first and the last value, as the rows may be apart)
        lo, hi = zip(*((p + min(0, (T - 1) * s) * x.element_size(), p + (max(0, (T - 1) * s) + H * D) * x.element_size())
                       for p, s in ((px, xs), (py, ys))))
        if lo[0] < hi[1] and lo[1] < hi[0] and not _columns_apart(px, xs, py, ys, H * D, x.element_size()):
            raise ValueError("out overlaps x without being x")
    st = _q.lib().qwam_rope(ctypes.byref(c), T, bool(inverse), px, xs, py, ys, _q._stream_ptr(stream))
    _q._check("qwam_rope", st)
    _q._written(out)
    return y


def _columns_apart(p: int, s: int, q: int, t: int, width: int, size: int) -> bool:
    """Whether rows of `width` values `s` apart from p, and the same from q, are other columns of one matrix."""
    if s != t or s == 0:
        return False
    gap = (q - p) % (abs(s) * size)
    return width * size <= gap <= (abs(s) - width) * size


class _Rope(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, positions, plan, inverse):
        ctx.save_for_backward(positions, plan.inv_freq, plan.axis)
        ctx.kept = (plan.interleaved, inverse)
        return _rope(x, positions, plan, inverse, None, None)

    @staticmethod
    def backward(ctx, dy):
        positions, inv_freq, axis = ctx.saved_tensors
        interleaved, inverse = ctx.kept
        return rope(dy.contiguous(), positions, RopePlan(inv_freq, axis, interleaved), inverse=not inverse), None, None, None


def rope(x: torch.Tensor, positions: torch.Tensor, plan: RopePlan, *, inverse: bool = False, out: Optional[torch.Tensor] = None,
         stream=None) -> torch.Tensor:
    """qwam_rope: x bf16 or float32 [tokens][heads][dim] (tokens may be apart: queries and keys beside each other in a layer's
    output are one call) turned by positions (int32 or float32 [rows][axes]; token t has row t % rows, so samples on one
    grid share it) as the plan says.  `inverse` turns back, which is the gradient.  `out` gives the output and may be x
    itself.  Returns it; gradients of x of any order, no forward-mode tangents."""
    if stream is None:
        y = (_q._call or _q._native()).rope(x, positions, plan, inverse, out)
        if y is not None:
            if type(y) is int:
                _q._check("qwam_rope", y)
            return y
    if isinstance(plan, RopePlan):
        held = {"plan.inv_freq": plan.inv_freq, "plan.axis": plan.axis}
        _q._no_tangent("rope", x=x, out=out)
        _q._no_gradient("rope", positions=positions, out=out, **held)
        if torch.is_grad_enabled() and isinstance(x, torch.Tensor) and x.requires_grad:
            if out is not None or stream is not None:
                raise ValueError("rope under autograd takes neither out nor stream")
            return _Rope.apply(x, positions, plan, bool(inverse))
    return _rope(x, positions, plan, inverse, out, stream)
