"""Experts on rows where many experts have few rows each, so that small tiles are many: against the experts in 64 bits."""
import pytest
import torch

from test_gpu_rows import U16, U32, gen, make_blobs, make_rows, offsets_of, within

pytestmark = pytest.mark.gpu
COUNTS = [3, 0, 65, 1, 16, 17, 130, 33, 64, 0] * 10


@pytest.mark.parametrize("fmt,hidden,inter", [("int8", 2048, 72), ("int8", 1024, 200), ("bf16", 2048, 72)])
def test_many_experts_with_few_rows(lib, fmt, hidden, inter):
    g = gen(inter)
    n, tail = sum(COUNTS), 7
    blobs, dense = make_blobs(lib, g, fmt, len(COUNTS), hidden, inter)
    xs, scale, x = make_rows(g, fmt, n + tail, hidden)
    ys = lib.experts_rows(fmt, blobs, inter, xs, offsets_of(COUNTS), scale=scale)
    assert not ys[n:].any()
    at = 0
    for e, (c, (wg, wu, wd)) in enumerate(zip(COUNTS, dense)):
        r = x[at:at + c]
        a, b = r @ wg.t(), r @ wu.t()
        s = torch.sigmoid(a)
        h = a * s * b
        ref = h @ wd.t()
        # h: its rounding to bf16 and the sums behind it (slope of silu at most 1.1); then the second sum and the result's rounding
        dh = U16 * h.abs() + 64 * U32 * (1.1 * b.abs() * (r.abs() @ wg.abs().t()) + (a * s).abs() * (r.abs() @ wu.abs().t())) + 8 * U32 * h.abs()
        within(ys[at:at + c], ref, 1.01 * (dh @ wd.abs().t()) + 64 * U32 * (h.abs() @ wd.abs().t()) + 1.01 * U16 * ref.abs() + 1e-12, f"expert {e}")
        at += c
    assert torch.equal(ys, lib.experts_rows(fmt, blobs, inter, xs, offsets_of(COUNTS), scale=scale))
