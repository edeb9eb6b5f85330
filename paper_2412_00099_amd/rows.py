"""The operators on many rows, for tensors: PyTorch allocates the outputs and workspaces, the library computes.

Everything runs on the current stream of the tensors' device and returns at once.  Tensors that belong to another stream have
to be ready there first, and be kept, as with any operator of PyTorch.  Shapes, types and places are checked ahead of the library
(ValueError, in csrc/rows_torch.cpp, where the outputs are made, too), the rest by the library (MoEError).  Automatic
differentiation is the caller's (examples/moe_layer.py): the calls record nothing, and while gradients are being recorded they
refuse inputs that require one (ValueError); inputs with a tangent of the forward mode they refuse, too.
"""
from __future__ import annotations

from typing import NamedTuple

import torch

from . import binding as B

try:
    from . import _rows
except ImportError as e:
    raise ImportError(f"{e}: build with `python paper_2412_00099_amd/build.py`") from e

_rows.raise_as(B.MoEError)
_ROW_FMT = {torch.float32: B.MOE_R_FP32, torch.bfloat16: B.MOE_R_BF16, torch.int8: B.MOE_R_INT8}


class NormedRows(NamedTuple):
    h: torch.Tensor             # the residual stream after the addition; without y the tensor that was given, not a copy
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


def _fmt(dtype):
    fmt = _ROW_FMT.get(dtype)
    if fmt is None:
        raise ValueError(f"{dtype} is not among {tuple(_ROW_FMT)}")
    return fmt


def norm_rows(h, y=None, gain=None, *, eps=1e-6, out=torch.bfloat16) -> NormedRows:
    """h + y and its root-mean-square norm times gain, as `out`: float32, bfloat16, or int8 codes with a scale per row."""
    return NormedRows._make(_rows.norm_rows(h, y, gain, eps, _fmt(out)))


def norm_rows_backward(h, gain, rstd, dx, dh=None):
    """(gradient of the rows that were added, gradient of gain or None without one).  h, rstd: norm_rows' results; dx: gradient of
    x; dh: gradient of the sum itself.  (Without y, h is the caller's own tensor and has to hold the same values still.)"""
    return _rows.norm_rows_backward(h, gain, rstd, dx, dh)


def sort_tokens(ids, n_experts) -> TokenOrder:
    """ids [tokens, top_k] int32: the expert of each place; others than 0..n_experts-1 are places without one."""
    return TokenOrder._make(_rows.sort_tokens(ids, n_experts))


def gather_rows(x, order, scale=None):
    """(xs, its scales or None): the rows of x, and of scale if there is one, in the order of the experts."""
    return _rows.gather_rows(x, order.offsets, order.row_of, scale)


def combine_rows(ys, order, weight=None, base=None, out=None):
    """base + the weighted sum of each token's rows, as base's type (without base: `out`, or the type of ys)."""
    if out is torch.int8:
        raise ValueError("a sum of rows is no whole number")
    return _rows.combine_rows(ys, order.offsets, order.row_of, weight, base, -1 if out is None else _fmt(out))


def combine_rows_backward(dy, ys, order, weight=None):
    """(gradient of ys, gradient of weight or None without one)"""
    return _rows.combine_rows_backward(dy, ys, order.offsets, order.row_of, weight)


def _weight_fmt(weight_fmt):
    return B.WEIGHT_FMT[weight_fmt] if isinstance(weight_fmt, str) else weight_fmt


def experts_rows(weight_fmt, blobs, inter, xs, offsets, *, scale=None, keep=False):
    """The SwiGLU experts on sorted rows.  blobs [n_experts, ...]: packed experts ('bf16' or 'int8'), as bytes or bfloat16;
    offsets: a TokenOrder's.  keep: returns (ys, KeptExperts) for the backward, else ys."""
    ys, h, gu = _rows.experts_rows(_weight_fmt(weight_fmt), blobs, inter, xs, offsets, scale, keep)
    return (ys, KeptExperts(h, gu)) if keep else ys


def experts_rows_backward(weight_fmt, blobs, inter, xs, offsets, kept, dys, *, rows=True, weights=True):
    """(gradient of xs, gradient of the blobs in their layout), each None where it is not wanted."""
    return _rows.experts_rows_backward(_weight_fmt(weight_fmt), blobs, inter, xs, offsets, kept.h, kept.gu, dys, rows, weights)
