"""The operators on many rows, for tensors: PyTorch allocates the outputs and workspaces, the library computes.

Everything runs on the current stream of the tensors' device and returns at once.  Tensors that belong to another stream have
to be ready there first, and be kept, as with any operator of PyTorch.  Shapes and types are checked here, the rest by the
library (MoEError).
"""
from __future__ import annotations

from typing import NamedTuple

import torch

from . import binding as B

_ROW_FMT = {torch.float32: B.MOE_R_FP32, torch.bfloat16: B.MOE_R_BF16, torch.int8: B.MOE_R_INT8}


class NormedRows(NamedTuple):
    h: torch.Tensor             # the residual stream after the addition
    x: torch.Tensor             # its norm, or 8-bit codes
    scale: torch.Tensor | None  # of 8-bit codes: one per row
    rstd: torch.Tensor          # 1 / sqrt(mean h^2 + eps) of each row, for the backward


class TokenOrder(NamedTuple):
    offsets: torch.Tensor   # [n_experts + 1]: expert e has rows offsets[e] .. offsets[e + 1] - 1
    row_of: torch.Tensor    # [tokens, top_k]: row of each place, -1: none
    entry_of: torch.Tensor  # [tokens * top_k]: place of each row, -1: a row of nobody


class KeptExperts(NamedTuple):
    """What the backward of the experts needs of the forward."""

    h: torch.Tensor
    gu: torch.Tensor


_FLOATS = (torch.float32, torch.bfloat16)
_empty = torch.empty


def _ptr(t):
    return None if t is None else t.data_ptr()


def _fmt(t, allowed):
    if t.dtype not in allowed:
        raise ValueError(f"{t.dtype} is not among {allowed}")
    return _ROW_FMT[t.dtype]


def _rows(t, name):
    """A matrix whose rows are dense (they may lie apart); returns its stride."""
    if t.dim() != 2 or (t.stride(1) != 1 and t.shape[1] > 1):
        raise ValueError(f"{name} has to be a matrix with dense rows")
    return t.stride(0) if t.shape[0] > 1 else t.shape[1]


def _dense(t, shape, dtype, name):
    if t is not None and (t.shape != shape or not t.is_contiguous() or (dtype is not None and t.dtype != dtype)):
        raise ValueError(f"{name} has to be contiguous, {tuple(shape)}" + (f", {dtype}" if dtype else ""))


class _Call:
    """The GPU that all tensors are on, made current for the call, and its current stream."""

    __slots__ = ("at", "back")

    def __init__(self, t, *others):
        self.at = at = t.get_device()
        if at < 0:
            raise ValueError("the tensors have to be on a GPU")
        for o in others:
            if o is not None and o.get_device() != at:
                raise ValueError("all tensors have to be on one GPU")

    def __enter__(self):
        self.back = torch.cuda.current_device()
        if self.back != self.at:
            torch.cuda.set_device(self.at)
        # (the number itself: making a Stream object of it takes longer than some of the kernels)
        return torch._C._cuda_getCurrentRawStream(self.at)

    def __exit__(self, *_):
        if self.back != self.at:
            torch.cuda.set_device(self.back)


def norm_rows(h, y=None, gain=None, *, eps=1e-6, out=torch.bfloat16) -> NormedRows:
    """h + y and its root-mean-square norm times gain, as `out`: float32, bfloat16, or int8 codes with a scale per row."""
    h_fmt, h_stride = _fmt(h, _FLOATS), _rows(h, "h")
    n, d = h.shape
    y_fmt, y_stride = h_fmt, d
    if y is not None:
        y_fmt, y_stride = _fmt(y, _FLOATS), _rows(y, "y")
        if y.shape != h.shape:
            raise ValueError("y has to have the shape of h")
    _dense(gain, (d,), torch.float32, "gain")
    if out not in _ROW_FMT:
        raise ValueError(f"{out} is not among {tuple(_ROW_FMT)}")
    with _Call(h, y, gain) as s:
        dev = h.device
        h_out = h if y is None else _empty((n, d), dtype=h.dtype, device=dev)
        x = _empty((n, d), dtype=out, device=dev)
        rstd = _empty(n, dtype=torch.float32, device=dev)
        scale = _empty(n, dtype=torch.float32, device=dev) if out is torch.int8 else None
        B.moe_norm_rows(h.data_ptr(), h_fmt, h_stride, _ptr(y), y_fmt, y_stride, _ptr(gain), eps, n, d,
                        None if y is None else h_out.data_ptr(), x.data_ptr(), _ROW_FMT[out], _ptr(scale), rstd.data_ptr(), s)
    return NormedRows(h_out, x, scale, rstd)


def norm_rows_backward(h, gain, rstd, dx, dh=None):
    """(gradient of the rows that were added, gradient of gain or None without one).  h, rstd: norm_rows' results; dx: gradient of
    x; dh: gradient of the sum itself."""
    h_fmt, x_fmt = _fmt(h, _FLOATS), _fmt(dx, _FLOATS)
    n, d = h.shape
    _dense(h, (n, d), None, "h")
    _dense(dx, (n, d), None, "dx")
    _dense(dh, (n, d), h.dtype, "dh")
    _dense(gain, (d,), torch.float32, "gain")
    _dense(rstd, (n,), torch.float32, "rstd")
    with _Call(h, gain, rstd, dx, dh) as s:
        out = _empty((n, d), dtype=h.dtype, device=h.device)
        dgain = torch.empty_like(gain) if gain is not None else None
        need = B.moe_norm_rows_backward_bytes(n, d) if gain is not None else 0
        work = _empty(need, dtype=torch.uint8, device=h.device) if need else None
        B.moe_norm_rows_backward(h.data_ptr(), h_fmt, _ptr(gain), rstd.data_ptr(), dx.data_ptr(), x_fmt, _ptr(dh), n, d,
                                 out.data_ptr(), _ptr(dgain), _ptr(work), need, s)
    return out, dgain


def sort_tokens(ids, n_experts) -> TokenOrder:
    """ids [tokens, top_k] int32: the expert of each place; others than 0..n_experts-1 are places without one."""
    if ids.dim() != 2:
        raise ValueError("ids has to be [tokens, top_k]")
    t, k = ids.shape
    _dense(ids, (t, k), torch.int32, "ids")
    with _Call(ids) as s:
        dev = ids.device
        offsets = _empty(n_experts + 1, dtype=torch.int32, device=dev)
        row_of, entry_of = _empty((t, k), dtype=torch.int32, device=dev), _empty(t * k, dtype=torch.int32, device=dev)
        need = B.moe_sort_tokens_bytes(t, k, n_experts)
        work = _empty(need, dtype=torch.uint8, device=dev) if need else None
        B.moe_sort_tokens(ids.data_ptr(), t, k, n_experts, offsets.data_ptr(), row_of.data_ptr(), entry_of.data_ptr(), _ptr(work),
                          need, s)
    return TokenOrder(offsets, row_of, entry_of)


def _order(order):
    t, k = order.row_of.shape
    e = order.offsets.shape[0] - 1
    _dense(order.row_of, (t, k), torch.int32, "row_of")
    _dense(order.offsets, (e + 1,), torch.int32, "offsets")
    return t, k, e


def gather_rows(x, order, scale=None):
    """(xs, its scales or None): the rows of x, and of scale if there is one, in the order of the experts."""
    t, k, e = _order(order)
    fmt, stride = _fmt(x, _ROW_FMT), _rows(x, "x")
    d = x.shape[1]
    if x.shape[0] != t:
        raise ValueError("x has to have a row for each token")
    _dense(scale, (t,), torch.float32, "scale")
    with _Call(x, scale, order.row_of, order.offsets) as s:
        xs = _empty((t * k, d), dtype=x.dtype, device=x.device)
        xs_scale = _empty(t * k, dtype=torch.float32, device=x.device) if scale is not None else None
        B.moe_gather_rows(x.data_ptr(), fmt, stride, _ptr(scale), order.row_of.data_ptr(), order.offsets.data_ptr(), t, k, e, d,
                          xs.data_ptr(), _ptr(xs_scale), s)
    return xs, xs_scale


def combine_rows(ys, order, weight=None, base=None, out=None):
    """base + the weighted sum of each token's rows, as base's type (without base: `out`, or the type of ys)."""
    t, k, _ = _order(order)
    d = ys.shape[1]
    _dense(ys, (t * k, d), None, "ys")
    _dense(weight, (t, k), torch.float32, "weight")
    _dense(base, (t, d), out, "base")
    with _Call(ys, weight, base, order.row_of) as s:
        y = _empty((t, d), dtype=base.dtype if base is not None else out or ys.dtype, device=ys.device)
        B.moe_combine_rows(ys.data_ptr(), _fmt(ys, _FLOATS), order.row_of.data_ptr(), _ptr(weight), _ptr(base), t, k, d,
                           y.data_ptr(), _fmt(y, _FLOATS), s)
    return y


def combine_rows_backward(dy, ys, order, weight=None):
    """(gradient of ys, gradient of weight or None without one)"""
    t, k, e = _order(order)
    d = dy.shape[1]
    _dense(dy, (t, d), None, "dy")
    _dense(ys, (t * k, d), None, "ys")
    _dense(weight, (t, k), torch.float32, "weight")
    with _Call(dy, ys, weight, order.row_of, order.offsets) as s:
        dys = torch.empty_like(ys)
        dweight = torch.empty_like(weight) if weight is not None else None
        B.moe_combine_rows_backward(dy.data_ptr(), _fmt(dy, _FLOATS), ys.data_ptr(), _fmt(ys, _FLOATS), order.row_of.data_ptr(),
                                    order.offsets.data_ptr(), _ptr(weight), t, k, e, d, dys.data_ptr(), _ptr(dweight), s)
    return dys, dweight


def _experts(weight_fmt, blobs, xs, offsets):
    """(format, experts, bytes from blob to blob, rows, hidden)"""
    wfmt = B.WEIGHT_FMT[weight_fmt] if isinstance(weight_fmt, str) else weight_fmt
    e = offsets.shape[0] - 1
    if not blobs.is_contiguous() or e < 1 or blobs.shape[0] != e:
        raise ValueError("blobs has to be contiguous, one blob for each expert of offsets")
    _dense(offsets, (e + 1,), torch.int32, "offsets")
    n, d = xs.shape
    _dense(xs, (n, d), torch.int8 if wfmt == B.MOE_W_INT8_PC else torch.bfloat16, "xs")
    return wfmt, e, blobs.nbytes // e, n, d


def experts_rows(weight_fmt, blobs, inter, xs, offsets, *, scale=None, keep=False):
    """The SwiGLU experts on sorted rows.  blobs [n_experts, ...]: packed experts ('bf16' or 'int8'); offsets: a TokenOrder's.
    keep: returns (ys, KeptExperts) for the backward, else ys."""
    wfmt, e, stride, n, d = _experts(weight_fmt, blobs, xs, offsets)
    _dense(scale, (n,), torch.float32, "scale")
    with _Call(xs, blobs, offsets, scale) as s:
        dev, pitch = xs.device, (inter + 63) // 64 * 64
        h = _empty((n, pitch), dtype=torch.bfloat16, device=dev)
        gu = _empty((n, 2, pitch), dtype=torch.float32, device=dev) if keep else None
        ys = _empty((n, d), dtype=torch.bfloat16, device=dev)
        B.moe_experts_rows(wfmt, d, inter, e, blobs.data_ptr(), stride, xs.data_ptr(), _ptr(scale), offsets.data_ptr(), n,
                           h.data_ptr(), _ptr(gu), ys.data_ptr(), s)
    return (ys, KeptExperts(h, gu)) if keep else ys


def experts_rows_backward(weight_fmt, blobs, inter, xs, offsets, kept, dys, *, rows=True, weights=True):
    """(gradient of xs, gradient of the blobs in their layout), each None where it is not wanted."""
    wfmt, e, stride, n, d = _experts(weight_fmt, blobs, xs, offsets)
    pitch = (inter + 63) // 64 * 64
    _dense(dys, (n, d), torch.bfloat16, "dys")
    _dense(kept.h, (n, pitch), torch.bfloat16, "kept.h")
    _dense(kept.gu, (n, 2, pitch), torch.float32, "kept.gu")
    with _Call(xs, blobs, offsets, dys, kept.h, kept.gu) as s:
        dgu = _empty((n, 2, pitch), dtype=torch.bfloat16, device=xs.device)
        dxs = torch.empty_like(xs) if rows else None
        dblobs = torch.empty_like(blobs) if weights else None
        B.moe_experts_rows_backward(wfmt, d, inter, e, blobs.data_ptr(), stride, xs.data_ptr(), offsets.data_ptr(), n,
                                    kept.h.data_ptr(), kept.gu.data_ptr(), dys.data_ptr(), dgu.data_ptr(), _ptr(dxs), _ptr(dblobs), s)
    return dxs, dblobs
