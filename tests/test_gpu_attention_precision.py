"""How near attention's results come to what the rounding of the results alone leaves.

The bounds of test_gpu_attention.py are worst cases of single elements; here are errors of whole tensors relative to their size, on
inputs that make a part of the arithmetic show:  r is the error of the exact result rounded to bf16.  An independent error of the same
size makes it 1.41 r.
"""
import math

import pytest
import torch

from test_gpu_attention import BF16, DEV, I8, gen, ints, normal, paged, paged_reference, reference, starts

pytestmark = pytest.mark.gpu


def error(got, want):
    return float((got.double() - want).norm() / want.norm())


def of_rounding(want):
    return error(want.to(BF16), want)


@pytest.mark.parametrize("dim", [64, 96, 128])
@pytest.mark.parametrize("each,keys,heads", [
    ([60] * 5, [64] * 5, 2),        # the forward's keys divided among wavefronts, the gradient's not
    ([60] * 5, [64] * 5, 40),       # whole tiles
    ([60], [1600], 2)])             # shares of the keys, in both
def test_gradients_of_scores_that_cancel(lib, dim, each, keys, heads):
    """Queries of zeros: P is 1 / n, and exact.  The keys have c times as much in common as of their own, and the sum of a query's dz is 0:
    dq has the keys' own parts only, but an error of dz, or one of delta, their common part.
      dz in one part: its rounding is as large as r, times c in the common direction.  In two: 2^-17 of it times c, less than r / 16.
      y + low for delta: 2^-18.  y alone: an error of r |y||dy| in all of a query's dz, of |v||dy|, with |y| = |v| / sqrt(n).  Their sum over n keys
      has c r |v||dy| / sqrt(n) in the common direction, and dq's own parts are as |v||dy| / sqrt(n).
    So dq is within 1.05 r with what the forward keeps, and without it, or with dz in one part, near c r; 4 r tells them apart."""
    c = 16.0
    g = gen(dim + heads)
    nq, nk = sum(each), sum(keys)
    q = torch.zeros(nq, heads, dim, device=DEV, dtype=BF16)
    k = (c * normal(g, 1, 1, dim) + normal(g, nk, heads, dim)).to(BF16)
    v, dy = normal(g, nk, heads, dim, dtype=BF16), normal(g, nq, heads, dim, dtype=BF16)
    at = dict(k_offsets=ints(starts(keys)))
    offsets = ints(starts(each))
    y, kept = lib.attend_rows(q, k, v, offsets, keep=True, **at)
    want = reference(q, k, v, each, keys, 0, 0, dim ** -0.5, dy)
    r = of_rounding(want["dq"][0])
    with_low = error(lib.attend_rows_backward(q, k, v, offsets, y, kept, dy, **at)[0], want["dq"][0])
    without = error(lib.attend_rows_backward(q, k, v, offsets, y, kept._replace(low=None), dy, **at)[0], want["dq"][0])
    assert with_low <= 1.05 * r, (with_low, r)
    assert without >= 4 * with_low, (without, with_low)


def test_gradients_of_keys_that_not_all_queries_see(lib):
    """Sequences of 32: all of a tile is masked, and there dk takes dz in two parts.  Scores are near 0, so that P is near 1 / n; its
    rounding makes an error of delta of 0.00125 / sqrt(n) of dz, 0.17 of that squared on the whole (n from 1 to 32, weights 1 / n): 1.05 r.
    In one part dz's own rounding would come to it, as large as r: 1.4 r."""
    g = gen(51)
    each, heads, dim = [32] * 60, 4, 64
    n = sum(each)
    q, k = normal(g, n, heads, dim, std=0.1, dtype=BF16), normal(g, n, heads, dim, std=0.5, dtype=BF16)
    v, dy = normal(g, n, heads, dim, dtype=BF16), normal(g, n, heads, dim, dtype=BF16)
    offsets = ints(starts(each))
    y, kept = lib.attend_rows(q, k, v, offsets, keep=True)
    want = reference(q, k, v, each, each, 0, 0, dim ** -0.5, dy)["dk"][0]
    got = error(lib.attend_rows_backward(q, k, v, offsets, y, kept, dy)[1], want)
    assert got <= 1.2 * of_rounding(want), (got, of_rounding(want))


@pytest.mark.parametrize("each,keys,heads", [([300], None, 2), ([700], None, 48), ([40], [2000], 2)])
def test_the_sum_that_divides_is_of_rounded_exponentials(lib, each, keys, heads):
    """All values the same: their mean is that value whatever the exponentials' rounding, if it is in both sums.  y and what its rounding leaves
    are within 2^-12 of it (sums of up to 2000 terms in 32 bits, 2^-13.5 and 2^-14.5 at the worst); with the sum of the exponentials ahead
    of their rounding, whose error is up to 2^-9 and does not average out over the few keys that count, some row is 2^-11.2 off."""
    g = gen(52 + heads)
    nk, dim = sum(keys or each), 64
    q, k = normal(g, sum(each), heads, dim, std=2.0, dtype=BF16), normal(g, nk, 1, dim, dtype=BF16)
    v = normal(g, 1, 1, dim, dtype=BF16).expand(nk, 1, dim).contiguous()
    y, kept = lib.attend_rows(q, k, v, ints(starts(each)), k_offsets=ints(starts(keys or each)), keep=True)
    off = (y.double() + kept.low.double() - v[0].double()).abs() / v[0].double().abs()
    assert float(off.max()) <= 2.0 ** -12, math.log2(float(off.max()))


@pytest.mark.parametrize("cache", [BF16, I8])
@pytest.mark.parametrize("lengths", [[700, 90, 333], [9000, 4000]])
def test_exponentials_over_pages_keep_16_bits(lib, cache, lengths):
    """Two parts of an exponential leave 2^-16 of it at most, which does not show beside y's own rounding; with one the error
    is 1.16 r over 700 keys and 1.24 r over 9000 (the same arithmetic in 64 bits with that rounding)."""
    g = gen(53)
    kv, dim = 4, 128
    values, pages, scales, table = paged(g, lengths, kv, dim, 16, cache)
    q = normal(g, len(lengths), 32, dim, std=2.0, dtype=BF16)
    want = paged_reference(q, values, 0, 0, dim ** -0.5)[0]
    got = error(lib.attend_pages(q, *pages, table, ints(lengths), *scales), want)
    assert got <= 1.05 * of_rounding(want), (got, of_rounding(want))
