"""Attention beside the experts, for tensors: of packed sequences (a prompt, a training batch) with its gradients, and of one new
token per sequence over a cache of pages.

Called as the operators on many rows are (rows.py): on the current stream of the tensors' device, returning at once, checks ahead of
the library (ValueError, in csrc/attend_torch.cpp) and in it (MoEError), nothing recorded for automatic differentiation.  Rows are
bfloat16 [tokens, heads, dim]; token and head strides are free (multiples of 16 bytes), so that q, k and v may be parts of one
projection's rows.  A query at position p sees key j if j <= p and, with a window, j > p - window or j < sinks.
"""
from __future__ import annotations

from typing import NamedTuple

import torch

from .rows import _rows


class PagePlan(NamedTuple):
    offsets: torch.Tensor    # [sequences + 1]: the new tokens of sequence i are rows offsets[i] .. offsets[i + 1] - 1
    slots: torch.Tensor      # [n_tokens]: where each row goes in the cache, -1: nowhere
    positions: torch.Tensor  # [n_tokens]: its position in its sequence, -1 behind the last sequence
    lengths: torch.Tensor    # [sequences]: tokens in the cache once these are stored
    used: torch.Tensor       # [1]: how far the free pages are used up; more than there are: some tokens got no page


class KeptAttention(NamedTuple):
    """What the backward of attend_rows needs of the forward, beside y."""

    lse: torch.Tensor         # [heads, rows]: log of the sums of exponentials
    low: torch.Tensor | None  # [rows, heads, dim]: what the rounding of y leaves


def plan_pages(have, more, table, free, page, n_tokens, *, used=None) -> PagePlan:
    """Pages for `more` new tokens of sequences that have `have` (int32 [sequences]), taken from `free` (int32, page ids) from
    element `used` (int32 [1], None: the first) on, and written into `table` (int32 [sequences, pages]) in place.  n_tokens: rows of
    slots and positions, as many as all new tokens or more.  A caller who gets pages back writes their ids ahead of free[used]
    and takes their number off `used`."""
    return PagePlan._make(_rows.plan_pages(have, more, table, free, page, n_tokens, used))


def store_pages(k, v, slots, k_pages, v_pages, k_scale=None, v_scale=None) -> None:
    """The rows of k and v (bfloat16 or float32) into their slots (int32, all different; -1: none) of the cache [pages, heads, page,
    dim], in place: bfloat16, or int8 codes with float32 scales [pages, heads, page]."""
    _rows.store_pages(k, v, slots, k_pages, v_pages, k_scale, v_scale)


def attend_pages(q, k_pages, v_pages, table, lengths, k_scale=None, v_scale=None, *, scale=None, window=0, sinks=0):
    """y [sequences, heads, dim]: attention of the last token of each sequence, q's row, over its `lengths` tokens (int32) in the
    pages of `table`.  Length 0: zeros.  scale: of the scores, 1 / sqrt(dim) without it."""
    return _rows.attend_pages(q, k_pages, v_pages, table, lengths, k_scale, v_scale, scale, window, sinks)


def attend_rows(q, k, v, offsets, *, k_offsets=None, scale=None, window=0, sinks=0, keep=False):
    """y [rows, heads, dim]: causal attention within each sequence, rows offsets[i] .. offsets[i + 1] - 1 of q over rows k_offsets[i] ..
    k_offsets[i + 1] - 1 of k and v (None: the same rows); the queries are the last rows of their sequence.  keep: returns (y,
    KeptAttention) for the backward, else y."""
    y, lse, low = _rows.attend_rows(q, k, v, offsets, k_offsets, scale, window, sinks, keep)
    return (y, KeptAttention(lse, low)) if keep else y


def attend_rows_backward(q, k, v, offsets, y, kept, dy, *, k_offsets=None, scale=None, window=0, sinks=0):
    """(gradient of q, of k, of v); y, kept: attend_rows' results with the same arguments; dy dense."""
    return _rows.attend_rows_backward(q, k, v, offsets, y, kept.lse, kept.low, dy, k_offsets, scale, window, sinks)
