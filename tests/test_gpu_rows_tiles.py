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


MIDDLE = [120, 97, 0, 128, 200, 33, 161, 64, 130, 70] * 8  # about a hundred rows an expert


@pytest.mark.parametrize("fmt,hidden,inter", [("bf16", 1024, 130), ("int8", 1024, 136)])
def test_many_experts_with_a_hundred_rows(lib, fmt, hidden, inter):
    g = gen(inter + 1)
    n, tail = sum(MIDDLE), 3
    blobs, dense = make_blobs(lib, g, fmt, len(MIDDLE), hidden, inter)
    xs, scale, x = make_rows(g, fmt, n + tail, hidden)
    off = offsets_of(MIDDLE)
    kept = None
    if fmt == "bf16":
        ys, kept = lib.experts_rows(fmt, blobs, inter, xs, off, keep=True)
        dys = xs.roll(1, 0).contiguous()
        dxs, dblobs = lib.experts_rows_backward(fmt, blobs, inter, xs, off, kept, dys)
        dw = dblobs.view(torch.bfloat16).view(len(MIDDLE), inter, 3, hidden)
        assert torch.equal(ys, lib.experts_rows(fmt, blobs, inter, xs, off)) and not dxs[n:].any()
    else:
        ys = lib.experts_rows(fmt, blobs, inter, xs, off, scale=scale)
    assert not ys[n:].any()
    at = 0
    for e, (c, (wg, wu, wd)) in enumerate(zip(MIDDLE, dense)):
        r = x[at:at + c]
        a, b = r @ wg.t(), r @ wu.t()
        s = torch.sigmoid(a)
        h = a * s * b
        ref = h @ wd.t()
        dh = U16 * h.abs() + 64 * U32 * (1.1 * b.abs() * (r.abs() @ wg.abs().t()) + (a * s).abs() * (r.abs() @ wu.abs().t())) + 8 * U32 * h.abs()
        within(ys[at:at + c], ref, 1.01 * (dh @ wd.abs().t()) + 64 * U32 * (h.abs() @ wd.abs().t()) + 1.01 * U16 * ref.abs() + 1e-12, f"expert {e}")
        if kept is not None and c:
            leaves = [v.clone().requires_grad_() for v in (r, wg, wu, wd)]
            y = (torch.nn.functional.silu(leaves[0] @ leaves[1].t()) * (leaves[0] @ leaves[2].t())) @ leaves[3].t()
            grads = torch.autograd.grad(y, leaves, dys[at:at + c].double())
            # (six roundings to bf16 on the way of a gradient at most)
            for got, want in zip((dxs[at:at + c], dw[e, :, 0], dw[e, :, 1], dw[e, :, 2].t()), grads):
                assert float((got.double() - want).norm() / want.norm()) <= 6 * U16
        at += c


@pytest.mark.parametrize("fmt,hidden,each", [("bf16", 2048, 470), ("int8", 1024, 830)])
def test_many_experts_with_many_rows(lib, fmt, hidden, each):
    inter, experts = 72, 40
    g = gen(each)
    counts = [each + (17 * e) % 61 - 30 for e in range(experts)]
    n, tail = sum(counts), 4
    blobs, dense = make_blobs(lib, g, fmt, experts, hidden, inter)
    xs, scale, x = make_rows(g, fmt, n + tail, hidden)
    off = offsets_of(counts)
    dxs = None
    if fmt == "bf16":
        ys, kept = lib.experts_rows(fmt, blobs, inter, xs, off, keep=True)
        dys = xs.roll(1, 0).contiguous()
        dxs, _ = lib.experts_rows_backward(fmt, blobs, inter, xs, off, kept, dys, weights=False)
        assert not dxs[n:].any()
    else:
        ys = lib.experts_rows(fmt, blobs, inter, xs, off, scale=scale)
    assert not ys[n:].any()
    at = 0
    for e, (c, (wg, wu, wd)) in enumerate(zip(counts, dense)):
        r = x[at:at + c]
        a, b = r @ wg.t(), r @ wu.t()
        s = torch.sigmoid(a)
        h = a * s * b
        ref = h @ wd.t()
        dh = U16 * h.abs() + 64 * U32 * (1.1 * b.abs() * (r.abs() @ wg.abs().t()) + (a * s).abs() * (r.abs() @ wu.abs().t())) + 8 * U32 * h.abs()
        within(ys[at:at + c], ref, 1.01 * (dh @ wd.abs().t()) + 64 * U32 * (h.abs() @ wd.abs().t()) + 1.01 * U16 * ref.abs() + 1e-12, f"expert {e}")
        if dxs is not None:
            leaf = r.clone().requires_grad_()
            y = (torch.nn.functional.silu(leaf @ wg.t()) * (leaf @ wu.t())) @ wd.t()
            want, = torch.autograd.grad(y, leaf, dys[at:at + c].double())
            assert float((dxs[at:at + c].double() - want).norm() / want.norm()) <= 6 * U16
        at += c
