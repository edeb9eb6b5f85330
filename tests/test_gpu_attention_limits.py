"""Attention and the cache's pages at the largest counts that they take, with no sequence at all, and with the largest and smallest values
of rows that go into 8 bits.  Bounds: test_gpu_attention.py."""
import pytest
import torch

from test_gpu_attention import BF16, DEV, F32, I8, close, coded, gen, ints, normal, paged, paged_reference, plan_by_hand, reference, starts, up

pytestmark = pytest.mark.gpu
MOST = 16384


@pytest.mark.parametrize("each,keys,heads,kv,dim,window,sinks,ahead,behind", [
    ([], None, 4, 2, 64, 0, 0, 0, 300),
    ([], [], 4, 2, 64, 0, 0, 0, 3000),
    ([70], None, 256, 256, 128, 0, 0, 0, 0),
    ([150, 3], None, 256, 1, 64, 0, 0, 0, 0),
    ([40, 300], [50, 300], 255, 3, 8, 70, 3, 0, 0),
    ([0] * 9000 + [130] + [0] * 7382 + [33], None, 4, 1, 64, 0, 0, 7, 9),
    ([1 if i % 300 == 0 else 0 for i in range(MOST)], None, 1, 1, 16, 0, 0, 0, 0),
    ([0] * (MOST - 1) + [300], [1 if i % 500 == 0 else 0 for i in range(MOST - 1)] + [300], 2, 1, 64, 10, 3, 0, 0)], ids=lambda c: str(c)[:20])
def test_rows(lib, each, keys, heads, kv, dim, window, sinks, ahead, behind):
    g, kk = gen(5), each if keys is None else keys
    a, b = ahead + sum(each), ahead + sum(kk)
    q, dy = normal(g, a + behind, heads, dim, std=2.0, dtype=BF16), normal(g, a + behind, heads, dim, dtype=BF16)
    k, v = normal(g, b + behind, kv, dim, dtype=BF16), normal(g, b + behind, kv, dim, dtype=BF16)
    offsets = ints([ahead + x for x in starts(each)])
    kw = dict(k_offsets=None if keys is None else ints([ahead + x for x in starts(kk)]), window=window, sinks=sinks)
    y, kept = lib.attend_rows(q, k, v, offsets, keep=True, **kw)
    grads = lib.attend_rows_backward(q, k, v, offsets, y, kept, dy, **kw)
    want = reference(q[ahead:a], k[ahead:b], v[ahead:b], each, kk, window, sinks, dim ** -0.5, dy[ahead:a])
    for got, name, end in zip((y, *grads), ("y", "dq", "dk", "dv"), (a, a, b, b)):
        assert not got[:ahead].any() and not got[end:].any(), name
        if end > ahead:
            close(got[ahead:end], *want[name], name)


@pytest.mark.parametrize("cache", [BF16, I8])
@pytest.mark.parametrize("lengths,heads,kv,dim,window,sinks,some", [
    ([40, 3000, 0], 256, 256, 64, 0, 0, [0, 1, 2]),
    ([40, 3000, 0], 256, 1, 128, 0, 0, [0, 1, 2]),
    ([3000 if i % 4000 == 7 else i % 3 for i in range(MOST)], 17, 1, 64, 100, 3, [0, 1, 2, 7, 8, 4007, MOST - 1])], ids=lambda c: str(c)[:20])
def test_pages(lib, cache, lengths, heads, kv, dim, window, sinks, some):
    g = gen(6)
    values, pages, scales, table = paged(g, lengths, kv, dim, 16, cache)
    q = normal(g, len(lengths), heads, dim, std=2.0, dtype=BF16)
    y = lib.attend_pages(q, *pages, table, ints(lengths), *scales, window=window, sinks=sinks)
    close(y[some], *paged_reference(q[some], [values[i] for i in some], window, sinks, dim ** -0.5), "y")


def test_plan(lib):
    g = torch.Generator().manual_seed(3)
    have, more = torch.randint(0, 40, (MOST,), generator=g).tolist(), torch.randint(0, 30, (MOST,), generator=g).tolist()
    table = [[i * 5 + j if j < up(h, 16) else -7 for j in range(5)] for i, h in enumerate(have)]
    free = list(range(100000, 160000))
    want = plan_by_hand(have, more, table, free, 11, 16, sum(more) + 5)
    t = ints(table)
    got = lib.plan_pages(ints(have), ints(more), t, ints(free), 16, sum(more) + 5, used=ints([11]))
    for what, a, b in zip(("table", "offsets", "slots", "positions", "lengths", "used"), (t, *got), want):
        assert a.tolist() == b, what


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_codes_of_the_largest_and_smallest_rows(lib, dtype):
    """Largest values from 2^-99 (a little above the 1e-30 below which codes are 0) to the largest finite ones, whose reciprocals are subnormal."""
    g = gen(8)
    tops = torch.tensor([2.0 ** e * 1.3 for e in (-99, -98, -60, 0, 60, 124, 125, 126, 127)] + [2.0 ** 128 * (1 - 2.0 ** -8), 1e-31, 1e-40], device=DEV, dtype=torch.float64)
    x = torch.rand(12, 2, 40, 64, generator=g, device=DEV, dtype=torch.float64) * 2 - 1
    x[..., 0] = 1.0
    x[:, :, 1, 1:] = (torch.arange(63, device=DEV) * 2 - 63 + 0.0) / 254  # (halves between codes, where they are held exactly)
    x = (x * tops[:, None, None, None]).to(dtype)
    assert bool(torch.isfinite(x).all())
    pages = [torch.full((1, 40, 16, 64), 9, dtype=I8, device=DEV) for _ in range(2)]
    scales = [torch.full((1, 40, 16), 5.0, device=DEV) for _ in range(2)]
    lib.store_pages(x[:, 0], x[:, 1], ints(list(range(12))), *pages, *scales)
    for w in range(2):
        codes, scale = coded(x[:, w])
        assert torch.equal(pages[w][0, :, :12].transpose(0, 1), codes)
        assert bool(((scales[w][0, :, :12].t() - scale).abs() <= 2.0 ** -23 * scale).all())
        assert bool((pages[w][0, :, 12:] == 9).all())
