"""Attention and the cache's pages against plain forms in 64 bits.

Whole numbers have to be equal.  Everything else is held to bounds that are computed with it, element by element.  U is the most
that a rounding to bf16 takes, relative to the value (2^-8).  Scores are sums of dim products in 32 bits, off by at most E =
(dim + 8) 2^-24 sum |q k| scale, so that an exponential is off by a share of 2 E (its own and that of the largest), and so is their
sum.  With A = sum P |v|:
  y   U |y| + (U + 4 E + 2^-16) A: its own rounding, that of P (over pages P keeps 16 bits and more: 2^-16 instead of U), the scores,
      and the sums over keys in 32 bits, of exponentials of 2^-20 and of up to 2048 terms
  dv  likewise, with sum P |dy| for A
  dq  U |dq| + scale sum_j |k_j| (U |dz_j| + P_j (U |dy||y| + (4 E + 2^-16) (|dy||v_j| + |dy||y|))): the rounding of dz, that of y in
      delta, and the scores' errors; dk likewise with |q|.  (1 + 2 U) on top for products of two of these.
"""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF16, F32, I8, I32 = torch.bfloat16, torch.float32, torch.int8, torch.int32
U = 2.0 ** -8
S = 2.0 ** -16


def gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def normal(g, *shape, std=1.0, dtype=F32):
    return (torch.randn(*shape, generator=g, device=DEV) * std).to(dtype)


def ints(v):
    return torch.tensor(v, dtype=I32, device=DEV)


def starts(each):
    at = [0]
    for n in each:
        at.append(at[-1] + n)
    return at


def up(a, b):
    return -(-a // b)


def close(got, want, bound, what):
    got = got.double()
    assert got.shape == want.shape
    assert bool(torch.isfinite(got).all()), what
    over = (got - want).abs() - bound * (1 + 2 * U)
    assert float(over.max()) <= 0, (what, float(over.max()), int(over.argmax()), float(((got - want).abs() / bound.clamp(min=1e-300)).max()))


def visible(nq, nk, window, sinks):
    p, j = torch.arange(nk - nq, nk, device=DEV)[:, None], torch.arange(nk, device=DEV)[None]
    ok = j <= p
    return ok if window == 0 else ok & ((j > p - window) | (j < sinks))


def one_head(q, k, v, ok, scale, dy=None, p_round=U):
    """of one head in 64 bits: y and its bound, and with dy the gradients and theirs"""
    dim = q.shape[1]
    z = (q @ k.t()) * scale
    e = torch.where(ok, (q.abs() @ k.abs().t()) * scale, 0.0)
    E = (dim + 8) * 2.0 ** -24 * (float(e.max()) if e.numel() else 0.0)
    p = torch.where(ok.any(1, keepdim=True), torch.softmax(z.masked_fill(~ok, -math.inf), 1), 0.0).nan_to_num(0.0)
    y = p @ v
    out = dict(y=(y, U * y.abs() + (p_round + 4 * E + S) * (p @ v.abs())))
    if dy is not None:
        a = (dy.abs() * y.abs()).sum(1, keepdim=True)
        dz = p * (dy @ v.t() - (dy * y).sum(1, keepdim=True))
        off = U * dz.abs() + p * (U * a + (4 * E + S) * (dy.abs() @ v.abs().t() + a))
        dv, dq, dk = p.t() @ dy, scale * (dz @ k), scale * (dz.t() @ q)
        out.update(dv=(dv, (U + 4 * E + S) * (p.t() @ dy.abs())), dq=(dq, scale * (off @ k.abs())), dk=(dk, scale * (off.t() @ q.abs())))
    return out


def reference(q, k, v, each, keys, window, sinks, scale, dy=None):
    """{name: (value, bound)} of packed sequences; rows of no sequence are zeros"""
    G = q.shape[1] // k.shape[1]
    names = dict(y=q) if dy is None else dict(y=q, dq=q, dk=k, dv=k)
    out = {n: [torch.zeros(t.shape, device=DEV, dtype=torch.float64) for _ in range(2)] for n, t in names.items()}
    tq = tk = 0
    for nq, nk in zip(each, keys):
        ok = visible(nq, nk, window, sinks)
        if nq and nk:
            for h in range(q.shape[1]):
                rows, cols = slice(tq, tq + nq), slice(tk, tk + nk)
                one = one_head(q[rows, h].double(), k[cols, h // G].double(), v[cols, h // G].double(), ok, scale, None if dy is None else dy[rows, h].double())
                for n, parts in one.items():
                    at = (rows, h) if n in ("y", "dq") else (cols, h // G)
                    for to, x in zip(out[n], parts):
                        to[at] += x
        tq, tk = tq + nq, tk + nk
    for n in out:
        if n != "y":
            out[n][1] += U * out[n][0].abs()
    return out


# ---- packed sequences --------------------------------------------------------------------------------------
ROWS = [
    # each, keys (None: the same), heads, kv, dim, window, sinks
    ([1], None, 1, 1, 64, 0, 0),
    ([1], None, 4, 2, 128, 0, 0),
    ([64], None, 2, 2, 128, 0, 0),
    ([333], None, 4, 4, 128, 0, 0),
    ([129, 0, 1, 255, 31], None, 4, 2, 64, 0, 0),
    ([5, 700, 130], None, 6, 2, 80, 0, 0),
    ([200, 67], None, 3, 1, 8, 0, 0),
    ([190], None, 2, 1, 72, 0, 0),
    ([300, 300], None, 8, 8, 128, 0, 0),
    ([500, 3, 64], None, 4, 2, 128, 100, 0),
    ([500, 3, 64], None, 4, 2, 128, 100, 5),
    ([700], None, 2, 1, 64, 1, 0),
    ([700], None, 2, 1, 64, 1, 1),
    ([700, 90], None, 2, 2, 96, 64, 130),
    ([260], None, 16, 1, 128, 33, 64),
    ([400], None, 2, 2, 128, 1 << 30, 3),
    ([400], None, 2, 2, 128, (1 << 31) - 1, (1 << 31) - 1),
    ([10, 1, 77], [400, 300, 77], 4, 2, 128, 0, 0),
    ([10, 1, 200], [400, 300, 900], 4, 4, 64, 150, 7),
    ([50, 130, 0, 9], [20, 7, 40, 0], 4, 2, 128, 0, 0),  # queries ahead of the first key, keys without queries, no keys
    ([50, 300], [20, 100], 2, 1, 64, 16, 2),
    ([3] * 70 + [200], None, 2, 1, 32, 0, 0),            # more sequences than lanes
    ([2] * 300 + [900, 5, 130], None, 16, 1, 64, 0, 0),  # ... and than threads
    ([2500, 700], None, 16, 1, 128, 0, 0),               # few heads of k: their queries are cut into pieces
    ([2500, 0, 701], None, 12, 2, 80, 200, 5),
    ([100, 1500], [2000, 1500], 8, 1, 96, 0, 0),
]


def rows_case(case, extra=0):
    each, keys, heads, kv, dim, window, sinks = case
    g = gen(len(each) * 1000 + sum(each) + dim + window % 97)
    keys = keys or each
    q = normal(g, sum(each) + extra, heads, dim, std=2.0, dtype=BF16)
    both = normal(g, sum(keys) + extra, 2, kv, dim, dtype=BF16)
    dy = normal(g, sum(each) + extra, heads, dim, dtype=BF16)
    return q, both[:, 0], both[:, 1], dy, keys


@pytest.mark.parametrize("case", ROWS, ids=str)
def test_rows(lib, case):
    each, given, heads, kv, dim, window, sinks = case
    q, k, v, dy, keys = rows_case(case)
    kw = dict(k_offsets=ints(starts(keys)) if given else None, window=window, sinks=sinks)
    offsets = ints(starts(each))
    y, kept = lib.attend_rows(q, k, v, offsets, keep=True, **kw)
    want = reference(q, k, v, each, keys, window, sinks, dim ** -0.5, dy)
    close(y, *want["y"], "y")
    grads = lib.attend_rows_backward(q, k, v, offsets, y, kept, dy, **kw)
    for n, got in zip(("dq", "dk", "dv"), grads):
        close(got, *want[n], n)
    assert torch.equal(lib.attend_rows(q, k, v, offsets, **kw), y)
    for a, b in zip(grads, lib.attend_rows_backward(q, k, v, offsets, y, kept, dy, **kw)):
        assert torch.equal(a, b)
    # without what the rounding of y leaves: within the same bounds
    for n, got in zip(("dq", "dk", "dv"), lib.attend_rows_backward(q, k, v, offsets, y, kept._replace(low=None), dy, **kw)):
        close(got, *want[n], n)


# ---- plan --------------------------------------------------------------------------------------------------
def plan_by_hand(have, more, table, free, used, page, n_tokens):
    table, width = [list(r) for r in table], len(table[0]) if table else 0
    offsets, slots, positions, lengths = [0], [], [], []
    for row, h, m in zip(table, (max(v, 0) for v in have), (max(v, 0) for v in more)):
        for j in range(min(up(h, page), width), min(up(h + m, page), width)):
            row[j] = free[used] if 0 <= used < len(free) else -1
            used += 1
        for pos in range(h, h + m):
            id_ = row[pos // page] if pos // page < width else -1
            slots.append(id_ * page + pos % page if id_ >= 0 else -1)
            positions.append(pos)
        offsets.append(offsets[-1] + m)
        lengths.append(h + m)
    pad = [-1] * n_tokens
    return table, offsets, (slots + pad)[:n_tokens], (positions + pad)[:n_tokens], lengths, [used]


@pytest.mark.parametrize("seqs,longest,new,page,spare,used", [
    (1, 0, 1, 16, 0, None), (1, 15, 1, 16, 5, None), (1, 16, 1, 16, 5, 0), (3, 100, 40, 16, 0, 2), (8, 1000, 1, 32, 3, 1), (70, 300, 90, 64, 0, None),
    (5, 50, 3000, 16, 0, 7), (300, 90, 20, 16, -40, 0), (1500, 40, 3, 16, 4, 3), (2500, 20, 9, 1024, -1000, None), (2, 5000, 5000, 256, 0, 0)])
def test_plan(lib, seqs, longest, new, page, spare, used):
    g = torch.Generator().manual_seed(seqs + longest)
    have = torch.randint(-2, longest + 1, (seqs,), generator=g).tolist()
    more = torch.randint(-1, new + 1, (seqs,), generator=g).tolist()
    have[-1], more[0] = longest, new
    width = max(1, up(longest + new, page) - (1 if seqs == 3 else 0))  # (with three the table is too narrow for the longest)
    need = sum(up(max(h, 0) + max(m, 0), page) - up(max(h, 0), page) for h, m in zip(have, more))
    pages = torch.randperm(seqs * width + need + 50, generator=g).tolist()
    table = [[pages.pop() if j < up(max(h, 0), page) else -7 for j in range(width)] for h in have]
    free = pages[:max(1, need + spare + (used or 0))]
    for n_tokens in (sum(max(m, 0) for m in more) + 13, max(1, sum(max(m, 0) for m in more) // 2)):
        want = plan_by_hand(have, more, table, free, used or 0, page, n_tokens)
        t = ints(table)
        got = lib.plan_pages(ints(have), ints(more), t, ints(free), page, n_tokens, used=None if used is None else ints([used]))
        for what, a, b in zip(("table", "offsets", "slots", "positions", "lengths", "used"), (t, *got), want):
            assert a.dtype == I32 and a.tolist() == b, what


def test_plan_of_numbers_that_pass_32_bits(lib):
    big = (1 << 31) - 1
    t = torch.full((3, 4), -1, dtype=I32, device=DEV)
    p = lib.plan_pages(ints([big, 5, 0]), ints([big, big, 3]), t, ints([1 << 28, 9, 4, 6]), 16, 40)
    assert p.lengths.tolist() == [big, big, 3] and p.offsets.tolist() == [0, big, big, big]
    assert p.slots.tolist() == [-1] * 40  # (the first sequence's tokens are beyond its row of the table)
    assert p.positions.tolist() == [big] * 40
    # the second has a page already, which is not in the table; it takes three, the third one
    assert t.tolist() == [[-1] * 4, [-1, 1 << 28, 9, 4], [6, -1, -1, -1]] and p.used.tolist() == [4]


def test_plan_of_nothing(lib):
    empty = ints([])
    p = lib.plan_pages(empty, empty, torch.empty(0, 5, dtype=I32, device=DEV), empty, 16, 3, used=ints([2]))
    assert p.offsets.tolist() == [0] and p.slots.tolist() == [-1] * 3 and p.positions.tolist() == [-1] * 3 and p.used.tolist() == [2]
    t = torch.empty(2, 0, dtype=I32, device=DEV)
    p = lib.plan_pages(ints([3, 0]), ints([1, 2]), t, empty, 16, 3)
    assert p.offsets.tolist() == [0, 1, 3] and p.slots.tolist() == [-1] * 3 and p.positions.tolist() == [3, 0, 1] and p.used.tolist() == [0]


# ---- store -------------------------------------------------------------------------------------------------
def coded(x):
    """codes and scales of the last dimension, in 64 bits"""
    x = x.double()
    top = x.abs().amax(-1, keepdim=True)
    ok = torch.isfinite(top) & (top >= 1e-30)
    codes = torch.where(ok, torch.round(127.0 * x / torch.where(ok, top, 1.0)), 0.0).nan_to_num(0.0)
    scale = torch.where(torch.isfinite(top), torch.where(ok, top / 127.0, 0.0), math.nan)
    return codes.to(I8), scale[..., 0]


@pytest.mark.parametrize("rows,kv,dim,page,apart", [(1, 1, 8, 16, 0), (7, 2, 64, 16, 0), (300, 3, 128, 32, 16), (1000, 1, 72, 1024, 0), (33, 8, 24, 64, 32),
                                                    (5000, 2, 96, 128, 0), (64, 5, 120, 16, 0)])
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("cache", [BF16, I8])
def test_store(lib, rows, kv, dim, page, apart, dtype, cache):
    g = gen(rows + dim)
    n = up(rows, page) + 3
    size = kv * page * dim
    pools = [torch.full((n, size + apart), 77, device=DEV).to(cache) for _ in range(2)]
    pages = [p[:, :size].view(n, kv, page, dim) for p in pools]
    scales = [torch.full((n, kv, page), 5.0, device=DEV) for _ in range(2)] if cache == I8 else [None, None]
    x = normal(g, rows, 2, kv, dim, dtype=dtype)
    x[0, 0, 0] = 0
    if rows > 6:
        x[1, 0, 0, 1], x[2, 1, 0, 0], x[3, 0, 0, 2] = math.inf, math.nan, 254.0  # (254: bf16 values half way between two codes)
        x[3, 0, 0, 3:] = torch.arange(dim - 3, device=DEV) - dim // 2
        x[4] = x[4] * 1e-34 if dtype == F32 else x[4]
    slots = torch.randperm(n * page, generator=g, device=DEV)[:rows].int()
    slots[rows // 2] = -1
    if rows > 6:
        slots[-1], slots[-2], slots[-3] = n * page, (1 << 31) - 1, -(1 << 31)
    want = [p.clone() for p in pages]
    want_scales = [s.clone() if s is not None else None for s in scales]
    there = (slots >= 0) & (slots < n * page)
    at = slots[there].long()
    for w, (to, sc) in enumerate(zip(want, want_scales)):
        if cache == BF16:
            to[at // page, :, at % page] = x[there][:, w].to(BF16)
        else:
            codes, scale = coded(x[there][:, w])
            to[at // page, :, at % page] = codes
            sc[at // page, :, at % page] = scale.float()
    lib.store_pages(x[:, 0], x[:, 1], slots, *pages, *scales)
    for got, ref in zip(pages, want):
        assert torch.equal(torch.nan_to_num(got.float(), 1e9), torch.nan_to_num(ref.float(), 1e9))
    for got, ref in zip(scales, want_scales):
        if got is not None:
            # (a scale is a quotient in 32 bits: half a step)
            assert torch.equal(got.isnan(), ref.isnan())
            assert bool(((got - ref).abs() <= 2.0 ** -23 * ref.abs()).logical_or(ref.isnan()).all())
    for p in pools:
        assert bool((p[:, size:].float() == 77).all())


# ---- one new token over pages ------------------------------------------------------------------------------
PAGED = [
    # lengths, heads, kv, dim, page, window, sinks
    ([1], 1, 1, 64, 16, 0, 0),
    ([0, 1, 2, 15, 16, 17, 31, 32, 33], 2, 2, 128, 16, 0, 0),
    ([777], 16, 16, 128, 16, 0, 0),
    ([64, 500, 0, 1000], 8, 2, 128, 64, 0, 0),
    ([300, 40], 12, 1, 64, 32, 0, 0),
    ([300, 0, 41], 17, 1, 128, 16, 0, 0),   # more heads than a product has columns
    ([90, 400], 40, 1, 96, 16, 0, 0),
    ([333, 1, 90], 6, 2, 72, 16, 0, 0),
    ([200, 100], 3, 3, 8, 16, 0, 0),
    ([1500, 40, 700], 4, 2, 80, 128, 0, 0),
    ([1500, 40, 700], 8, 2, 128, 16, 100, 0),
    ([1500, 40, 700, 0, 104], 8, 2, 128, 16, 100, 4),
    ([1500, 64, 33], 2, 1, 64, 32, 1, 0),
    ([1500, 64, 33], 2, 1, 64, 32, 1, 70),
    ([3000, 2999], 4, 4, 24, 1024, 1000, 33),
    ([3000, 200], 4, 4, 64, 16, (1 << 31) - 1, 5),
    ([20000], 8, 2, 128, 16, 0, 0),
    ([5] * 150 + [0] * 20 + [70] * 90, 4, 2, 64, 16, 0, 0),
]


def paged(g, lengths, kv, dim, page, cache, bad=math.nan, apart=0, spare=2):
    """(k and v in 64 bits for each sequence, pages, scales, table): what no sequence has is `bad`"""
    there = [up(n, page) for n in lengths]
    n = sum(there) + spare
    size = kv * page * dim
    pools = [torch.full((n, size + apart), bad, device=DEV).to(BF16) if cache == BF16 else torch.full((n, size + apart), 99, dtype=I8, device=DEV) for _ in range(2)]
    pages = [p[:, :size].view(n, kv, page, dim) for p in pools]
    scales = [torch.full((n, kv, page), bad, device=DEV) for _ in range(2)] if cache == I8 else [None, None]
    ids = torch.randperm(n, generator=g, device=DEV).tolist()
    table = torch.full((len(lengths), max(there + [1]) + 1), -1, dtype=I32, device=DEV)
    table[:, -1] = 1 << 30
    values = []
    for i, m in enumerate(lengths):
        mine = [ids.pop() for _ in range(there[i])]
        table[i, :there[i]] = ints(mine)
        pos = torch.arange(m, device=DEV)
        p = ints(mine).long()[pos // page] if m else pos
        one = []
        for w in range(2):
            x = normal(g, m, kv, dim)
            if cache == I8:
                codes, scale = coded(x)
                scales[w][p, :, pos % page] = scale.float()
                x = codes.double() * scale.float().double()[..., None]
                pages[w][p, :, pos % page] = codes
            else:
                x = x.to(BF16)
                pages[w][p, :, pos % page] = x
            one.append(x.double())
        values.append(one)
    return values, pages, scales, table


def paged_reference(q, values, window, sinks, scale):
    out = [torch.zeros(q.shape, device=DEV, dtype=torch.float64) for _ in range(2)]
    for i, (k, v) in enumerate(values):
        if k.shape[0] == 0:
            continue
        ok = visible(1, k.shape[0], window, sinks)
        for h in range(q.shape[1]):
            kv = h // (q.shape[1] // k.shape[1])
            one = one_head(q[i, h, None].double(), k[:, kv], v[:, kv], ok, scale, p_round=S)["y"]
            for to, x in zip(out, one):
                to[i, h] = x[0]
    return out


@pytest.mark.parametrize("cache", [BF16, I8])
@pytest.mark.parametrize("case", PAGED, ids=lambda c: str(c)[:60])
def test_pages(lib, case, cache):
    lengths, heads, kv, dim, page, window, sinks = case
    g = gen(len(lengths) + sum(lengths) + dim)
    values, pages, scales, table = paged(g, lengths, kv, dim, page, cache, apart=32)
    q = normal(g, len(lengths), heads + 2, dim, std=2.0, dtype=BF16)[:, 1:-1]
    got = lib.attend_pages(q, *pages, table, ints(lengths), *scales, window=window, sinks=sinks)
    close(got, *paged_reference(q, values, window, sinks, dim ** -0.5), "y")
    for i, n in enumerate(lengths):
        assert n or not got[i].any()
    again = lib.attend_pages(q, *pages, table, ints(lengths), *scales, window=window, sinks=sinks)
    assert torch.equal(got, again)


def test_pages_that_are_not_there(lib):
    """Pages of the table that are none hide their tokens; a length beyond the table sees what the table has; a window's earlier pages may have been given away."""
    g = gen(5)
    lengths, page = [200, 130, 90], 16
    values, pages, _, table = paged(g, lengths, 2, 64, page, BF16)
    q = normal(g, 3, 4, 64, dtype=BF16)
    table[0, 3], table[0, 7], table[1, :9], table[2, 0] = -1, pages[0].shape[0], -5, -(1 << 31)
    seen = [torch.ones(n, dtype=torch.bool, device=DEV) for n in lengths]
    seen[0][48:64] = False
    seen[0][112:128] = False
    seen[1][:] = False
    seen[2][:16] = False
    kept = [[x[ok] for x in one] for one, ok in zip(values, seen)]
    close(lib.attend_pages(q, *pages, table, ints(lengths)), *paged_reference(q, kept, 0, 0, 0.125), "missing")
    values, pages, _, table = paged(g, lengths, 2, 64, page, BF16)
    close(lib.attend_pages(q, *pages, table[:, :5].contiguous(), ints(lengths), scale=0.3), *paged_reference(q, [[x[:80] for x in one] for one in values], 0, 0, 0.3), "narrow")
    table[0, :10] = -1
    table[0, 0:1] = ints([0])
    y = lib.attend_pages(q, *pages, table, ints([200, -3, 0]), window=30)
    k, v = values[0]
    want = paged_reference(q[:1], [[k[-30:], v[-30:]]], 0, 0, 0.125)
    close(y[:1], *want, "window")
    assert not y[1:].any()
