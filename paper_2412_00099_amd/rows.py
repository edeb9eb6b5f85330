"""The operators on many rows, for tensors: PyTorch allocates the outputs and workspaces, the library computes.

Everything runs on the current stream of the tensors' device and returns at once.  Tensors that belong to another stream have
to be ready there first, and be kept, as with any operator of PyTorch.  Shapes and types are checked here, the rest by the
library (MoEError).
"""
from __future__ import annotations

from functools import lru_cache
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


_FLOATS = {torch.float32: B.MOE_R_FP32, torch.bfloat16: B.MOE_R_BF16}
# (sizes one by one: as a tuple they take a fifth longer)
_empty, _empty_like = torch.empty, torch.empty_like
# (the numbers themselves: making Stream and device objects of them takes longer than some of the kernels)
_current_device, _stream_of = torch._C._cuda_getDevice, torch._C._cuda_getCurrentRawStream


def _ptr(t):
    return None if t is None else t.data_ptr()


def _fmt(t, allowed):
    fmt = allowed.get(t.dtype)
    if fmt is None:
        raise ValueError(f"{t.dtype} is not among {tuple(allowed)}")
    return fmt


def _rows(t, name):
    """(rows, columns, stride) of a matrix whose rows are dense (they may lie apart)."""
    shape, stride = t.shape, t.stride()
    if len(shape) != 2 or (stride[1] != 1 and shape[1] > 1):
        raise ValueError(f"{name} has to be a matrix with dense rows")
    n, d = shape
    return n, d, stride[0] if n > 1 else d


def _dense(t, shape, dtype, name):
    if t is not None and (t.shape != shape or not t.is_contiguous() or (dtype is not None and t.dtype != dtype)):
        raise ValueError(f"{name} has to be contiguous, {tuple(shape)}" + (f", {dtype}" if dtype else ""))


def _on(t, *others):
    """The GPU that all of the tensors are on."""
    at = t.get_device()
    if at < 0:
        raise ValueError("the tensors have to be on a GPU")
    for o in others:
        if o is not None and o.get_device() != at:
            raise ValueError("all tensors have to be on one GPU")
    return at


def _elsewhere(at, f, *args, **kw):
    """f with GPU `at` as the current one"""
    with torch.cuda.device(at):
        return f(*args, **kw)


_backward_bytes = lru_cache(maxsize=256)(B.moe_norm_rows_backward_bytes)
_sort_bytes = lru_cache(maxsize=256)(B.moe_sort_tokens_bytes)


def norm_rows(h, y=None, gain=None, *, eps=1e-6, out=torch.bfloat16) -> NormedRows:
    """h + y and its root-mean-square norm times gain, as `out`: float32, bfloat16, or int8 codes with a scale per row."""
    h_fmt, (n, d, h_stride) = _fmt(h, _FLOATS), _rows(h, "h")
    y_fmt, y_stride = h_fmt, d
    if y is not None:
        y_fmt, (yn, yd, y_stride) = _fmt(y, _FLOATS), _rows(y, "y")
        if yn != n or yd != d:
            raise ValueError("y has to have the shape of h")
    _dense(gain, (d,), torch.float32, "gain")
    x_fmt = _ROW_FMT.get(out)
    if x_fmt is None:
        raise ValueError(f"{out} is not among {tuple(_ROW_FMT)}")
    at = _on(h, y, gain)
    if at != _current_device():
        return _elsewhere(at, norm_rows, h, y, gain, eps=eps, out=out)
    h_out = h if y is None else _empty_like(h) if h_stride == d else h.new_empty(n, d)
    x = _empty(n, d, dtype=out, device=h.device)
    rstd = _empty(n, dtype=torch.float32, device=h.device)
    scale = _empty_like(rstd) if out is torch.int8 else None
    B.moe_norm_rows(h.data_ptr(), h_fmt, h_stride, _ptr(y), y_fmt, y_stride, _ptr(gain), eps, n, d,
                    None if y is None else h_out.data_ptr(), x.data_ptr(), x_fmt, _ptr(scale), rstd.data_ptr(), _stream_of(at))
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
    at = _on(h, gain, rstd, dx, dh)
    if at != _current_device():
        return _elsewhere(at, norm_rows_backward, h, gain, rstd, dx, dh)
    out = _empty_like(h)
    dgain = _empty_like(gain) if gain is not None else None
    need = _backward_bytes(n, d) if gain is not None else 0
    work = _empty(need, dtype=torch.uint8, device=h.device) if need else None
    B.moe_norm_rows_backward(h.data_ptr(), h_fmt, _ptr(gain), rstd.data_ptr(), dx.data_ptr(), x_fmt, _ptr(dh), n, d,
                             out.data_ptr(), _ptr(dgain), _ptr(work), need, _stream_of(at))
    return out, dgain


def sort_tokens(ids, n_experts) -> TokenOrder:
    """ids [tokens, top_k] int32: the expert of each place; others than 0..n_experts-1 are places without one."""
    if ids.dim() != 2:
        raise ValueError("ids has to be [tokens, top_k]")
    t, k = ids.shape
    _dense(ids, (t, k), torch.int32, "ids")
    at = _on(ids)
    if at != _current_device():
        return _elsewhere(at, sort_tokens, ids, n_experts)
    offsets, row_of, entry_of = ids.new_empty(n_experts + 1), _empty_like(ids), ids.new_empty(t * k)
    need = _sort_bytes(t, k, n_experts)
    work = _empty(need, dtype=torch.uint8, device=ids.device) if need else None
    B.moe_sort_tokens(ids.data_ptr(), t, k, n_experts, offsets.data_ptr(), row_of.data_ptr(), entry_of.data_ptr(), _ptr(work), need,
                      _stream_of(at))
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
    fmt, (n, d, stride) = _fmt(x, _ROW_FMT), _rows(x, "x")
    if n != t:
        raise ValueError("x has to have a row for each token")
    _dense(scale, (t,), torch.float32, "scale")
    at = _on(x, scale, order.row_of, order.offsets)
    if at != _current_device():
        return _elsewhere(at, gather_rows, x, order, scale)
    xs = x.new_empty(t * k, d)
    xs_scale = scale.new_empty(t * k) if scale is not None else None
    B.moe_gather_rows(x.data_ptr(), fmt, stride, _ptr(scale), order.row_of.data_ptr(), order.offsets.data_ptr(), t, k, e, d,
                      xs.data_ptr(), _ptr(xs_scale), _stream_of(at))
    return xs, xs_scale


def combine_rows(ys, order, weight=None, base=None, out=None):
    """base + the weighted sum of each token's rows, as base's type (without base: `out`, or the type of ys)."""
    t, k, _ = _order(order)
    ys_fmt, d = _fmt(ys, _FLOATS), ys.shape[-1]
    _dense(ys, (t * k, d), None, "ys")
    _dense(weight, (t, k), torch.float32, "weight")
    _dense(base, (t, d), out, "base")
    at = _on(ys, weight, base, order.row_of)
    if at != _current_device():
        return _elsewhere(at, combine_rows, ys, order, weight, base, out)
    if base is not None:
        y = _empty_like(base)
    elif out is None or out is ys.dtype:
        y = ys.new_empty(t, d)
    else:
        y = _empty(t, d, dtype=out, device=ys.device)
    B.moe_combine_rows(ys.data_ptr(), ys_fmt, order.row_of.data_ptr(), _ptr(weight), _ptr(base), t, k, d, y.data_ptr(),
                       _fmt(y, _FLOATS), _stream_of(at))
    return y


def combine_rows_backward(dy, ys, order, weight=None):
    """(gradient of ys, gradient of weight or None without one)"""
    t, k, e = _order(order)
    d = dy.shape[-1]
    _dense(dy, (t, d), None, "dy")
    _dense(ys, (t * k, d), None, "ys")
    _dense(weight, (t, k), torch.float32, "weight")
    at = _on(dy, ys, weight, order.row_of, order.offsets)
    if at != _current_device():
        return _elsewhere(at, combine_rows_backward, dy, ys, order, weight)
    dys = _empty_like(ys)
    dweight = _empty_like(weight) if weight is not None else None
    B.moe_combine_rows_backward(dy.data_ptr(), _fmt(dy, _FLOATS), ys.data_ptr(), _fmt(ys, _FLOATS), order.row_of.data_ptr(),
                                order.offsets.data_ptr(), _ptr(weight), t, k, e, d, dys.data_ptr(), _ptr(dweight), _stream_of(at))
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
    at = _on(xs, blobs, offsets, scale)
    if at != _current_device():
        return _elsewhere(at, experts_rows, weight_fmt, blobs, inter, xs, offsets, scale=scale, keep=keep)
    dev, pitch = xs.device, (inter + 63) // 64 * 64
    h = _empty(n, pitch, dtype=torch.bfloat16, device=dev)
    gu = _empty(n, 2, pitch, dtype=torch.float32, device=dev) if keep else None
    ys = _empty(n, d, dtype=torch.bfloat16, device=dev)
    B.moe_experts_rows(wfmt, d, inter, e, blobs.data_ptr(), stride, xs.data_ptr(), _ptr(scale), offsets.data_ptr(), n,
                       h.data_ptr(), _ptr(gu), ys.data_ptr(), _stream_of(at))
    return (ys, KeptExperts(h, gu)) if keep else ys


def experts_rows_backward(weight_fmt, blobs, inter, xs, offsets, kept, dys, *, rows=True, weights=True):
    """(gradient of xs, gradient of the blobs in their layout), each None where it is not wanted."""
    wfmt, e, stride, n, d = _experts(weight_fmt, blobs, xs, offsets)
    pitch = (inter + 63) // 64 * 64
    _dense(dys, (n, d), torch.bfloat16, "dys")
    _dense(kept.h, (n, pitch), torch.bfloat16, "kept.h")
    _dense(kept.gu, (n, 2, pitch), torch.float32, "kept.gu")
    at = _on(xs, blobs, offsets, dys, kept.h, kept.gu)
    if at != _current_device():
        return _elsewhere(at, experts_rows_backward, weight_fmt, blobs, inter, xs, offsets, kept, dys, rows=rows, weights=weights)
    dgu = _empty(n, 2, pitch, dtype=torch.bfloat16, device=xs.device)
    dxs = _empty_like(xs) if rows else None
    dblobs = _empty_like(blobs) if weights else None
    B.moe_experts_rows_backward(wfmt, d, inter, e, blobs.data_ptr(), stride, xs.data_ptr(), offsets.data_ptr(), n, kept.h.data_ptr(),
                                kept.gu.data_ptr(), dys.data_ptr(), dgu.data_ptr(), _ptr(dxs), _ptr(dblobs), _stream_of(at))
    return dxs, dblobs
