"""The operators on many rows at the ends of what they take."""
import pytest
import torch

from test_gpu_rows import DEV, F32, U32, gen, normal, within

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
