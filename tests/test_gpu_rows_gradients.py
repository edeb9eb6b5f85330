"""Gradients of the experts on rows, element by element, and of the norm's gain from call to call.

Roundings to bf16 on the way of an element: H, the gradients of G and U, the result.  G and U themselves and all sums are in 32
bits: a sum over n values is a chain of n / 32 additions behind sums of 32, at most 69 additions here, each (and each truncation ahead
of it) off by u32 of the terms' sizes at most, so that 160 u32 of the sum of the sizes holds.  The functions of G and U in between
are a few roundings long: 16 u32 of their terms' sizes.  d silu / dg is 1.1 at most, its slope 0.5.
"""
import pytest
import torch

from test_gpu_rows import BF16, COUNTS, F32, MANY, U16, U32, gen, make_blobs, make_rows, normal, offsets_of, within
from test_gpu_rows_tiles import MIDDLE

pytestmark = pytest.mark.gpu
SUM, FEW, MORE = 160 * U32, 16 * U32, 1.02  # (MORE: products of two such errors)


def gradients(x, wg, wu, wd, dy):
    """(value, bound of its error) of dx, dgate, dup and of down's gradient as [inter, hidden], in 64 bits.  wd: [hidden, inter]."""
    a, b, dh = x @ wg.t(), x @ wu.t(), dy @ wd
    s = torch.sigmoid(a)
    h, slope = a * s * b, s * (1 + a * (1 - s))
    dg, du = dh * b * slope, dh * a * s
    off_a, off_b, off_dh = SUM * (x.abs() @ wg.abs().t()), SUM * (x.abs() @ wu.abs().t()), SUM * (dy.abs() @ wd.abs())
    off_h = U16 * h.abs() + 1.1 * b.abs() * off_a + (a * s).abs() * off_b + FEW * h.abs()
    off_dg = (U16 * dg.abs() + (b * slope).abs() * off_dh + (dh * slope).abs() * off_b + 0.5 * (dh * b).abs() * off_a
              + FEW * (dh * b).abs() * (1 + a.abs()))
    off_du = U16 * du.abs() + (a * s).abs() * off_dh + 1.1 * dh.abs() * off_a + FEW * du.abs()
    for ref, off, size in (
            (dg @ wg + du @ wu, off_dg @ wg.abs() + off_du @ wu.abs(), dg.abs() @ wg.abs() + du.abs() @ wu.abs()),
            (dg.t() @ x, off_dg.t() @ x.abs(), dg.abs().t() @ x.abs()),
            (du.t() @ x, off_du.t() @ x.abs(), du.abs().t() @ x.abs()),
            (h.t() @ dy, off_h.t() @ dy.abs(), h.abs().t() @ dy.abs())):
        yield ref, MORE * (off + SUM * size + U16 * ref.abs()) + 1e-12


SMALL = [(c, *s) for c in COUNTS for s in ((512, 64), (512, 1), (1024, 200), (2048, 129))]
LARGE = [(MANY, 1024, 1000), (MANY, 2048, 897), (MIDDLE, 1024, 130), ([440 + (17 * e) % 61 for e in range(40)], 2048, 72)]


@pytest.mark.parametrize("counts,hidden,inter", SMALL + LARGE)
def test_every_element_of_the_experts_gradients(lib, counts, hidden, inter):
    g = gen(sum(counts) + 3 * inter)
    n, tail = sum(counts), 3
    blobs, dense = make_blobs(lib, g, "bf16", len(counts), hidden, inter)
    xs, _, x = make_rows(g, "bf16", n + tail, hidden)
    dys = normal(g, n + tail, hidden, dtype=BF16)
    _, kept = lib.experts_rows("bf16", blobs, inter, xs, offsets_of(counts), keep=True)
    dxs, dblobs = lib.experts_rows_backward("bf16", blobs, inter, xs, offsets_of(counts), kept, dys)
    assert not dxs[n:].any()
    dw = dblobs.view(BF16).view(len(counts), inter, 3, hidden)
    at = 0
    for e, (c, w) in enumerate(zip(counts, dense)):
        if c == 0:
            assert not dw[e].any()
            continue
        mine = (dxs[at:at + c], dw[e, :, 0], dw[e, :, 1], dw[e, :, 2])
        for got, (ref, bound), what in zip(mine, gradients(x[at:at + c], *w, dys[at:at + c].double()), ("dx", "dgate", "dup", "ddown")):
            within(got, ref, bound, f"{what} of expert {e}")
        at += c


@pytest.mark.parametrize("hidden", [1, 100, 513, 1024, 2048, 3001, 8191, 8192])
@pytest.mark.parametrize("rows", [1, 7, 1100])
@pytest.mark.parametrize("ht,xt", [(F32, BF16), (BF16, F32), (F32, F32), (BF16, BF16)])
def test_gain_gradient_is_the_same_from_call_to_call(lib, hidden, rows, ht, xt):
    """Bit for bit, and whether or not the rows' own gradient is passed on."""
    g = gen(5 * hidden + rows)
    h, gain = normal(g, rows, hidden, dtype=ht, std=2.0), 1 + normal(g, hidden, std=0.2)
    dx, up = normal(g, rows, hidden, dtype=xt), normal(g, rows, hidden, dtype=ht)
    rstd = lib.norm_rows(h, gain=gain).rstd
    dh, dgain = lib.norm_rows_backward(h, gain, rstd, dx, up)
    again, dgain2 = lib.norm_rows_backward(h, gain, rstd, dx, up)
    _, without = lib.norm_rows_backward(h, gain, rstd, dx)
    assert torch.equal(dh, again) and torch.equal(dgain, dgain2) and torch.equal(dgain, without)
