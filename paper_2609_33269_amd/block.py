"""Python binding of what surrounds the layers in one token's step: the norms
around a block with its gate and residual scale, and the paged key-value cache
with the attention that reads it (include/qwam.h).  As in `qwam`, arguments are
checked here, every step runs in the library's HIP kernels, and there is no
fallback.

block_norm is differentiable: with an input that requires a gradient it records
block_norm_backward, so probe vectors can be back-propagated through the norms
between two layers (those through the layers themselves are the caller's, by
the float weights).  asp_matvec and the cache's calls have no gradient and
refuse inputs that require one.
"""

from __future__ import annotations

import ctypes
from dataclasses import dataclass
from typing import Optional

import torch

from . import qwam as _q

NORM_KINDS = {"rms": 0, "layer": 1}
CACHE_TYPES = {torch.bfloat16: 0, torch.float8_e4m3fn: 1}


# ---------------------------------------------------------------------------
# norms around a block
# ---------------------------------------------------------------------------

def _per_sample(t: Optional[torch.Tensor], name: str, S: int, D: int):
    """Pointer and sample stride of an optional bf16 [S][D] whose rows may be apart (a slice of a wider tensor)."""
    if t is None:
        return None, 0
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch.Tensor")
    if t.device.type != "cuda":
        raise ValueError(f"{name} must be a GPU tensor (got {t.device})")
    if t.dtype != torch.bfloat16:
        raise TypeError(f"{name} must be {torch.bfloat16} (got {t.dtype})")
    if tuple(t.shape) != (S, D):
        raise ValueError(f"{name} must have shape {(S, D)} (got {tuple(t.shape)})")
    if D > 1 and t.stride(1) != 1:
        raise ValueError(f"{name} must be contiguous along its rows")
    return t.data_ptr(), t.stride(0)


def _samples(gate, scale, shift) -> int:
    for name, t in (("gate", gate), ("scale", scale), ("shift", shift)):
        if t is not None:
            if not isinstance(t, torch.Tensor):
                raise TypeError(f"{name} must be a torch.Tensor")
            if t.dim() != 2:
                raise ValueError("gate, scale and shift have two dimensions (samples, width)")
            return t.shape[0]
    return 1


def _norm_struct(x, norm, eps, residual_scale, gate, post_norm, post_weight, weight, scale, shift, x_name="x"):
    if norm not in NORM_KINDS:
        raise ValueError(f"norm must be one of {sorted(NORM_KINDS)} (got {norm!r})")
    if not isinstance(x, torch.Tensor) or x.dim() != 2:
        raise ValueError(f"{x_name} must be a tensor of two dimensions (rows, width)")
    if x.dtype not in (torch.bfloat16, torch.float32):
        raise TypeError(f"{x_name} must be {torch.bfloat16} or {torch.float32} (got {x.dtype})")
    if post_weight is not None and not post_norm:
        raise ValueError("post_weight without post_norm")
    T, D = x.shape
    S = _samples(gate, scale, shift)
    c = _q.QwamNormC()
    c.T, c.D, c.S, c.kind, c.post, c.x_f32 = T, D, S, NORM_KINDS[norm], bool(post_norm), x.dtype == torch.float32
    c.eps, c.residual_scale = eps, residual_scale
    c.gate, c.gate_stride = _per_sample(gate, "gate", S, D)
    c.scale, c.scale_stride = _per_sample(scale, "scale", S, D)
    c.shift, c.shift_stride = _per_sample(shift, "shift", S, D)
    c.post_weight = None if post_weight is None else _q._req(post_weight, "post_weight", torch.bfloat16, (D,))
    c.weight = None if weight is None else _q._req(weight, "weight", torch.bfloat16, (D,))
    return c


def _forward(x, branch, norm, eps, residual_scale, gate, post_norm, post_weight, weight, scale, shift, out, stream):
    c = _norm_struct(x, norm, eps, residual_scale, gate, post_norm, post_weight, weight, scale, shift)
    T, D = x.shape
    px = _q._req(x, "x", x.dtype, (T, D))
    pb = None if branch is None else _q._req(branch, "branch", torch.bfloat16, (T, D))
    xo, h = (None, None) if out is None else out
    if branch is None:
        if xo is not None:
            raise ValueError("out[0] without a branch")
    elif xo is None:
        xo = _q._empty((T, D), x.dtype, x.device, stream)
    if h is None:
        h = _q._empty((T, D), torch.bfloat16, x.device, stream)
    st = _q.lib().qwam_block_norm(ctypes.byref(c), px, pb, None if xo is None else _q._req(xo, "out[0]", x.dtype, (T, D)),
                                  _q._req(h, "out[1]", torch.bfloat16, (T, D)), _q._stream_ptr(stream))
    _q._check("qwam_block_norm", st)
    return xo, h


class _BlockNorm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, branch, gate, post_weight, weight, scale, shift, norm, eps, residual_scale, post_norm):
        xo, h = _forward(x, branch, norm, eps, residual_scale, gate, post_norm, post_weight, weight, scale, shift, None, None)
        ctx.save_for_backward(x if branch is None else xo, branch, gate, post_weight, weight, scale, shift)
        ctx.kept = (norm, eps, residual_scale, post_norm)
        ctx.set_materialize_grads(False)      # the gradient of an unused output is None, not T x D zeros
        return xo, h

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dxo, dh):
        xo, branch, gate, post_weight, weight, scale, shift = ctx.saved_tensors
        norm, eps, residual_scale, post_norm = ctx.kept
        if dh is None:
            dh = torch.zeros(xo.shape, dtype=torch.bfloat16, device=xo.device)
        need = dict(zip(("x", "branch", "gate", "post_weight", "weight", "scale", "shift"), ctx.needs_input_grad))
        g = block_norm_backward(None if dxo is None else dxo.contiguous(), dh.contiguous(), xo, branch, norm=norm, eps=eps,
                                residual_scale=residual_scale, gate=gate, post_norm=post_norm, post_weight=post_weight,
                                weight=weight, scale=scale, shift=shift,
                                wanted=tuple("d" + n for n, w in need.items() if w))
        # (None too for a gate or post_weight that a norm without a branch does not read)
        like = lambda n, t: g["d" + n].to(t.dtype) if need[n] and g["d" + n] is not None else None  # noqa: E731
        return (g["dx"] if need["x"] else None, g.get("dbranch"), like("gate", gate), like("post_weight", post_weight),
                like("weight", weight), like("scale", scale), like("shift", shift), None, None, None, None)


def block_norm(x: torch.Tensor, branch: Optional[torch.Tensor] = None, *, norm: str = "rms", eps: float = 1e-6,
               residual_scale: float = 1.0, gate: Optional[torch.Tensor] = None, post_norm: bool = False,
               post_weight: Optional[torch.Tensor] = None, weight: Optional[torch.Tensor] = None,
               scale: Optional[torch.Tensor] = None, shift: Optional[torch.Tensor] = None, out=None, stream=None):
    """qwam_block_norm: what lies between two blocks.

        x' = residual_scale * x + gate * u,   u = branch, or N(branch) * post_weight with post_norm
        h  = N(x') * weight * (1 + scale) + shift

    x bf16 or float32 [T][D], branch bf16 [T][D]; gate, scale, shift bf16 [S][D] for S samples of T / S consecutive rows
    (their rows may be apart: a slice of a modulation's wider output); post_weight, weight bf16 [D].  Each of them may be
    None.  Returns (x' as x, h bf16); without a branch (the norm in front of the first block), (None, h) with x' = x.
    `out` = (x', h) gives the outputs; x' may be x itself.  Gradients as block_norm_backward's; no forward-mode tangents."""
    if stream is None and out is None:
        done = (_q._call or _q._native()).norm(x, branch, norm, eps, residual_scale, gate, post_norm, post_weight, weight, scale,
                                               shift)
        if done is not None:
            if type(done) is int:
                _q._check("qwam_block_norm", done)
            return done
    _q._no_tangent("block_norm", x=x, branch=branch, gate=gate, post_weight=post_weight, weight=weight, scale=scale, shift=shift)
    if torch.is_grad_enabled() and any(isinstance(t, torch.Tensor) and t.requires_grad
                                       for t in (x, branch, gate, post_weight, weight, scale, shift)):
        if out is not None or stream is not None:
            raise ValueError("block_norm under autograd takes neither out nor stream")
        return _BlockNorm.apply(x, branch, gate, post_weight, weight, scale, shift, norm, eps, residual_scale, post_norm)
    return _forward(x, branch, norm, eps, residual_scale, gate, post_norm, post_weight, weight, scale, shift, out, stream)


def block_norm_backward(dx_out: Optional[torch.Tensor], dh: torch.Tensor, x_out: torch.Tensor,
                        branch: Optional[torch.Tensor] = None, *, norm: str = "rms", eps: float = 1e-6,
                        residual_scale: float = 1.0, gate: Optional[torch.Tensor] = None, post_norm: bool = False,
                        post_weight: Optional[torch.Tensor] = None, weight: Optional[torch.Tensor] = None,
                        scale: Optional[torch.Tensor] = None, shift: Optional[torch.Tensor] = None, wanted=None, stream=None):
    """qwam_block_norm_backward: the gradients of block_norm at the stored x' (without a branch: x), from those of x'
    (None: none) and of h.  Returns a dict with dx (as x'), dbranch (bf16), and float32 dgate, dscale, dshift [S][D] and
    dpost_weight, dweight [D] for the parameters given (None for the others).  `wanted` limits the parameters' and the
    branch's gradients to those named.  What it returns is not differentiable further."""
    if stream is None and wanted is None:
        done = (_q._call or _q._native()).norm_backward(dx_out, dh, x_out, branch, norm, eps, residual_scale, gate, post_norm,
                                                        post_weight, weight, scale, shift)
        if done is not None:
            if type(done) is int:
                _q._check("qwam_block_norm_backward", done)
            return done
    _q._no_tangent("block_norm_backward", dx_out=dx_out, dh=dh, x_out=x_out, branch=branch, gate=gate, post_weight=post_weight,
                   weight=weight, scale=scale, shift=shift)
    c = _norm_struct(x_out, norm, eps, residual_scale, gate, post_norm, post_weight, weight, scale, shift, "x_out")
    T, D = x_out.shape
    dev = x_out.device
    pd = None if dx_out is None else _q._req(dx_out, "dx_out", x_out.dtype, (T, D))
    ph = _q._req(dh, "dh", torch.bfloat16, (T, D))
    px = _q._req(x_out, "x_out", x_out.dtype, (T, D))
    pb = None if branch is None else _q._req(branch, "branch", torch.bfloat16, (T, D))
    has = {"dbranch": branch is not None, "dgate": branch is not None and gate is not None,
           "dpost_weight": branch is not None and post_weight is not None, "dweight": weight is not None,
           "dscale": scale is not None, "dshift": shift is not None}
    g = {"dx": _q._empty((T, D), x_out.dtype, dev, stream)}
    for name, given in has.items():
        if not given or (wanted is not None and name not in wanted):
            g[name] = None
        elif name == "dbranch":
            g[name] = _q._empty((T, D), torch.bfloat16, dev, stream)
        else:
            g[name] = _q._empty((D,) if name in ("dweight", "dpost_weight") else (c.S, D), torch.float32, dev, stream)
    need = _q._need("qwam_block_norm_backward", _q.lib().qwam_block_norm_backward_workspace(ctypes.byref(c)))
    ws = _q._workspace(need, dev, stream)
    ptr = lambda n: None if g[n] is None else g[n].data_ptr()  # noqa: E731
    st = _q.lib().qwam_block_norm_backward(ctypes.byref(c), pd, ph, px, pb, ptr("dx"), ptr("dbranch"), ptr("dgate"),
                                           ptr("dscale"), ptr("dshift"), ptr("dpost_weight"), ptr("dweight"),
                                           None if ws is None else ws.data_ptr(), need, _q._stream_ptr(stream))
    _q._check("qwam_block_norm_backward", st)
    return g


# ---------------------------------------------------------------------------
# paged key-value cache
# ---------------------------------------------------------------------------

@dataclass
class PagedCache:
    """Keys and values in pages (include/qwam.h): position p of sequence s in row p % page of page table[s, p // page].

    k, v: bf16 or float8_e4m3fn [pages][heads][page][dim], equal strides, dim contiguous (any order of the others: pages
    that hold their rows first, or both of k and v, are views of this form).  table: int32 [sequences][width], entries
    outside the pages mean no page.  k_scale, v_scale: float32 [heads], with float8 pages (value = code * scale)."""
    k: torch.Tensor
    v: torch.Tensor
    table: torch.Tensor
    k_scale: Optional[torch.Tensor] = None
    v_scale: Optional[torch.Tensor] = None

    def _values(self) -> dict:
        return {"cache.k": self.k, "cache.v": self.v, "cache.k_scale": self.k_scale, "cache.v_scale": self.v_scale}

    def c_struct(self) -> "_q.QwamCacheC":
        for t, name in ((self.k, "k"), (self.v, "v")):
            if not isinstance(t, torch.Tensor):
                raise TypeError(f"{name} must be a torch.Tensor")
            if t.device.type != "cuda":
                raise ValueError(f"{name} must be a GPU tensor (got {t.device})")
            if t.dtype not in CACHE_TYPES or t.dtype != self.k.dtype:
                raise TypeError(f"{name} must be {torch.bfloat16} or {torch.float8_e4m3fn}, k and v alike (got {t.dtype})")
            if t.dim() != 4 or t.shape != self.k.shape:
                raise ValueError(f"{name} must have shape [pages][heads][page][dim], k and v alike (got {tuple(t.shape)})")
            if t.stride(3) != 1 or t.stride() != self.k.stride():
                raise ValueError(f"{name} must be contiguous along dim, with k's strides (got {t.stride()})")
        if not isinstance(self.table, torch.Tensor) or self.table.dim() != 2:
            raise ValueError("table must be a tensor of two dimensions (sequences, width)")
        c = _q.QwamCacheC()
        c.pages, c.heads, c.page_size, c.dim = self.k.shape
        c.type, (c.seqs, c.table_width) = CACHE_TYPES[self.k.dtype], self.table.shape
        c.page_stride, c.head_stride, c.row_stride = self.k.stride()[:3]
        c.k, c.v = self.k.data_ptr(), self.v.data_ptr()
        c.table = _q._req(self.table, "table", torch.int32, tuple(self.table.shape))
        if c.type:
            c.k_scale = _q._req(self.k_scale, "k_scale", torch.float32, (c.heads,))
            c.v_scale = _q._req(self.v_scale, "v_scale", torch.float32, (c.heads,))
        return c


def new_cache(pages: int, heads: int, dim: int, seqs: int, table_width: int, page: int = 64, dtype=torch.bfloat16,
              k_scale: Optional[torch.Tensor] = None, v_scale: Optional[torch.Tensor] = None, device="cuda") -> PagedCache:
    """An empty cache: zeroed pages, tables without pages."""
    z = lambda: torch.zeros((pages, heads, page, dim), dtype=torch.bfloat16, device=device).to(dtype)  # noqa: E731
    return PagedCache(z(), z(), torch.full((seqs, table_width), -1, dtype=torch.int32, device=device), k_scale, v_scale)


def _rows(t: torch.Tensor, name: str, shape) -> int:
    """Pointer of a bf16 [rows][heads][dim] whose rows may be apart (a slice of a layer's wider output)."""
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a torch.Tensor")
    if t.device.type != "cuda":
        raise ValueError(f"{name} must be a GPU tensor (got {t.device})")
    if t.dtype != torch.bfloat16:
        raise TypeError(f"{name} must be {torch.bfloat16} (got {t.dtype})")
    if tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name} must have shape {tuple(shape)} (got {tuple(t.shape)})")
    if (t.shape[2] > 1 and t.stride(2) != 1) or (t.shape[1] > 1 and t.stride(1) != t.shape[2]):
        raise ValueError(f"{name} must be contiguous along its heads")
    return t.data_ptr()


def kv_append(cache: PagedCache, k: torch.Tensor, v: torch.Tensor, seq: torch.Tensor, pos: torch.Tensor, stream=None) -> None:
    """qwam_kv_append: k, v bf16 [tokens][heads][dim] to position pos[t] of sequence seq[t] (int32 [tokens]), rounded to
    float8 where the pages are.  Tokens without a place (pos < 0, no page) are not stored.  There is no gradient: tensors
    that require one are refused where autograd records."""
    if stream is None:
        st = (_q._call or _q._native()).append(cache, k, v, seq, pos)
        if st is not None:
            _q._check("qwam_kv_append", st)
            return
    c = cache.c_struct()
    if not isinstance(k, torch.Tensor) or k.dim() != 3:
        raise ValueError("k must be a tensor of three dimensions (tokens, heads, dim)")
    n = k.shape[0]
    _q._no_gradient("kv_append", k=k, v=v, **cache._values())
    st = _q.lib().qwam_kv_append(ctypes.byref(c), n, _rows(k, "k", (n, c.heads, c.dim)), k.stride(0) if n > 1 else 0,
                                 _rows(v, "v", (n, c.heads, c.dim)), v.stride(0) if n > 1 else 0,
                                 _q._req(seq, "seq", torch.int32, (n,)), _q._req(pos, "pos", torch.int32, (n,)),
                                 _q._stream_ptr(stream))
    _q._check("qwam_kv_append", st)


def paged_attention(cache: PagedCache, q: torch.Tensor, lengths: torch.Tensor, *, starts: Optional[torch.Tensor] = None,
                    scale: Optional[float] = None, max_len: Optional[int] = None, out: Optional[torch.Tensor] = None,
                    stream=None) -> torch.Tensor:
    """qwam_paged_attention: one new token per sequence, q bf16 [sequences][q_heads][dim] -> out bf16 of the same shape.
    Sequence b sees positions starts[b] (0) to lengths[b] (int32 [sequences]); one that sees none gives zeros.  `scale`
    is dim ** -0.5 unless given.  `max_len` bounds the lengths (the table's reach unless given): the work is laid out
    for it, and positions past it are not seen.  There is no gradient, as for kv_append."""
    if stream is None:
        o = (_q._call or _q._native()).attention(cache, q, lengths, starts, scale, max_len, out)
        if o is not None:
            if type(o) is int:
                _q._check("qwam_paged_attention", o)
            return o
    c = cache.c_struct()
    if not isinstance(q, torch.Tensor) or q.dim() != 3:
        raise ValueError("q must be a tensor of three dimensions (sequences, heads, dim)")
    Hq = q.shape[1]
    shape = (c.seqs, Hq, c.dim)
    pq = _rows(q, "q", shape)
    _q._no_gradient("paged_attention", q=q, **cache._values())
    if max_len is None:
        max_len = c.table_width * c.page_size
    need = _q._need("qwam_paged_attention", _q.lib().qwam_paged_attention_workspace(ctypes.byref(c), Hq, max_len))
    o = _q._empty(shape, torch.bfloat16, q.device, stream) if out is None else out
    ws = _q._workspace(need, q.device, stream)
    st = _q.lib().qwam_paged_attention(
        ctypes.byref(c), Hq, pq, q.stride(0) if c.seqs > 1 else 0, _q._req(lengths, "lengths", torch.int32, (c.seqs,)),
        None if starts is None else _q._req(starts, "starts", torch.int32, (c.seqs,)), max_len,
        float(c.dim ** -0.5 if scale is None else scale), _q._req(o, "out", torch.bfloat16, shape),
        None if ws is None else ws.data_ptr(), need, _q._stream_ptr(stream))
    _q._check("qwam_paged_attention", st)
    return o
