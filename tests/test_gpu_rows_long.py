"""The operators on many rows at the ends of what they take: the most rows, and blobs whose offsets pass 31 bits."""
import pytest
import torch

from test_gpu_rows import BF16, DEV, F32, U16, U32, gen, normal, offsets_of, within
from test_gpu_rows_gradients import gradients

pytestmark = pytest.mark.gpu
MOST = (1 << 26) - 1


def test_norm_of_the_most_rows(lib):
    h = normal(gen(1), MOST, 1)
    n = lib.norm_rows(h, out=F32)
    rstd = (h.double().square() + 1e-6).rsqrt()
    within(n.rstd, rstd[:, 0], 64 * U32 * rstd[:, 0], "rstd")
    x = h.double() * rstd
    within(n.x, x, 64 * U32 * x.abs(), "x")


def test_order_of_the_most_places(lib):
    g = gen(2)
    ids = torch.randint(-1, 3, (MOST, 1), generator=g, device=DEV, dtype=torch.int32)  # (-1 and 2: no expert)
    o = lib.sort_tokens(ids, 2)
    flat = ids[:, 0]
    entry = torch.cat([(flat == e).nonzero()[:, 0] for e in (0, 1)])
    n = entry.numel()
    assert o.offsets.tolist() == [0, int((flat == 0).sum()), n]
    assert torch.equal(o.entry_of[:n].long(), entry) and bool((o.entry_of[n:] == -1).all())
    row = torch.full((MOST,), -1, device=DEV, dtype=torch.int32)
    row[entry] = torch.arange(n, device=DEV, dtype=torch.int32)
    assert torch.equal(o.row_of[:, 0], row)
    x, weight = normal(g, MOST, 1), torch.rand(MOST, 1, generator=g, device=DEV)
    xs, _ = lib.gather_rows(x, o)
    assert torch.equal(xs[:n], x[entry]) and not xs[n:].any()
    there = (row >= 0)[:, None]
    ref = torch.where(there, x.double() * weight.double(), 0.0)
    within(lib.combine_rows(xs, o, weight), ref, 2 * U32 * ref.abs(), "y")
    dys, dweight = lib.combine_rows_backward(x, xs, o, weight)
    within(dys[:n], ref[entry], 2 * U32 * ref[entry].abs(), "dys")
    assert not dys[n:].any()
    square = torch.where(there, x.double().square(), 0.0)
    within(dweight, square, 2 * U32 * square, "dweight")


def test_an_expert_of_four_gigabytes(lib):
    """One large tile of rows: offsets into the blob, its gradient and the kept sums pass 2^31 bytes."""
    hidden, inter, rows = 512, 1310719, 250
    g = gen(3)
    w = torch.empty(1, inter, 3, hidden, device=DEV, dtype=BF16)
    w.normal_(0.0, 0.05, generator=g)
    assert w.nbytes == lib.moe_blob_bytes(lib.MOE_W_BF16, hidden, inter) and w.nbytes > 0xefff0000
    xs, dys = normal(g, rows + 2, hidden, dtype=BF16), normal(g, rows + 2, hidden, dtype=BF16, std=0.01)
    ys, kept = lib.experts_rows("bf16", w, inter, xs, offsets_of([rows]), keep=True)
    dxs, dw = lib.experts_rows_backward("bf16", w, inter, xs, offsets_of([rows]), kept, dys)
    assert not ys[rows:].any() and not dxs[rows:].any()
    x, dy = xs[:rows].double(), dys[:rows].double()
    y, dx = torch.zeros_like(x), torch.zeros_like(x)
    for at in range(0, inter, 1 << 16):
        wg, wu, wd = w[0, at:at + (1 << 16)].double().unbind(1)
        a, b = x @ wg.t(), x @ wu.t()
        y += (torch.nn.functional.silu(a) * b) @ wd
        (one, _), *weights = gradients(x, wg, wu, wd.t(), dy)
        dx += one
        for i, (ref, bound) in enumerate(weights):
            within(dw[0, at:at + (1 << 16), i], ref, bound, f"records from {at} on, {i}")
    # (sums over 1.3 million records: as vectors, each row's and each column's; one rounding of the products or gradients that are
    # summed and one of the result, twice over)
    for got, ref in ((ys[:rows], y), (dxs[:rows], dx)):
        for dim in (0, 1):
            assert bool(((got.double() - ref).norm(dim=dim) <= 4 * U16 * ref.norm(dim=dim)).all())
