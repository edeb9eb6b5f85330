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
    ([i % 4 for i in range(3000)] + [400], None, 2, 1, 64, 0, 0),
    ([2] * 80 + [0, 70, 1], None, 1, 1, 64, 0, 0),
    ([0] * 70 + [130, 0, 257] + [0] * 5000, None, 2, 2, 72, 40, 2),
    ([2500, 700], None, 16, 1, 128, 0, 0),               # few heads of k: their queries are cut into pieces
    ([2500, 0, 701], None, 12, 2, 80, 200, 5),
    ([100, 1500], [2000, 1500], 8, 1, 96, 0, 0),
    ([100], [4000], 4, 2, 128, 0, 0),                    # few queries of many keys: the keys are cut into shares
    ([1, 0, 40, 3], [4500, 700, 1900, 0], 2, 1, 72, 0, 0),
    ([130, 6], [2900, 1300], 2, 2, 64, 1600, 5),
    ([130], [3001], 6, 1, 96, 1400, 130),
    ([1800], None, 1, 1, 80, 0, 0),
    ([1] + [0] * 70 + [90], [1000] * 71 + [40000], 1, 1, 16, 0, 0),
]


def rows_case(case, extra=0):
    each, keys, heads, kv, dim, window, sinks = case
    g = gen(len(each) * 1000 + sum(each) + dim + window % 97)
    keys = keys or each
    q = normal(g, sum(each) + extra, heads, dim, std=2.0, dtype=BF16)
    both = normal(g, sum(keys) + extra, 2, kv, dim, dtype=BF16)
    dy = normal(g, sum(each) + extra, heads, dim, dtype=BF16)
    return q, both[:, 0], both[:, 1], dy, keys


def many_heads(case):
    """The case with as many heads, in groups of the same size, as it takes for more than 128 workgroups of 128 queries: up to there
    the forward divides the keys among the wavefronts of a workgroup instead."""
    each, keys, heads, kv, dim, window, sinks = case
    times = up(129, (sum(each) // 128 + len(each) + 1) * heads)
    return each, keys, heads * times, kv * times, dim, window, sinks


@pytest.mark.parametrize("case", ROWS + [many_heads(c) for c in ROWS if len(c[0]) < 1000], ids=lambda c: str(c)[:90])
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


@pytest.mark.parametrize("window,sinks,dim", [(0, 0, 128), (0, 0, 64), (60, 0, 80), (60, 40, 128)])
@pytest.mark.parametrize("what", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("times", [1, 6])
def test_rows_that_are_not_seen_may_hold_anything(lib, window, sinks, dim, what, times):
    """Behind the last sequence, in another sequence, ahead of a window, and of the same sequence but later on."""
    g = gen(dim + window)
    each, H, KV = [300, 90], 4 * times, 2 * times
    q = normal(g, 400, H, dim, std=2.0, dtype=BF16)
    k, v = normal(g, 400, KV, dim, dtype=BF16), normal(g, 400, KV, dim, dtype=BF16)
    want = reference(q[:390], k[:390], v[:390], each, each, window, sinks, dim ** -0.5)["y"]
    q[390:], k[390:], v[390:] = what, what, what
    at = 133
    v[at, 0, 5] = what   # of one key: dim 5 of heads 0 and 1
    v[at + 1, 1] = what  # of the next one: all of heads 2 and 3
    k[at + 37, 1, 0] = math.nan
    y = lib.attend_rows(q, k, v, ints(starts(each)), window=window, sinks=sinks)
    assert not y[390:].any()
    clean = torch.ones(390, H, dim, dtype=torch.bool, device=DEV)
    ok = visible(300, 300, window, sinks)
    clean[:300][ok[:, at], 0:2, 5] = False
    clean[:300, 2:4][ok[:, at + 1] | ok[:, at + 37]] = False
    over = (y[:390].double() - want[0]).abs() - want[1] * (1 + 2 * U)
    assert float(torch.where(clean, over, -1.0).max()) <= 0  # (a comparison with NaN would be false)
    got = y[:300].float()
    assert bool(torch.isfinite(got[clean[:300]]).all())
    one = got[ok[:, at]][:, 0:2, 5]
    assert bool((one.isnan() if what != what else one == what).all())
    # (rows that see the NaN key are NaN, the others have the values' infinities)
    two = got[ok[:, at + 1] & ~ok[:, at + 37]][:, 2:4]
    assert bool((two.isnan() if what != what else two == what).all())
    assert bool(got[ok[:, at + 37]][:, 2:4].isnan().all())


@pytest.mark.parametrize("what", [math.nan, math.inf])
def test_shares_of_keys_that_are_not_seen(lib, what):
    """As above where the keys are cut into shares; rows of no sequence are zeros, and so is what sees no key."""
    g = gen(21)
    H, KV, dim, each, keys = 2, 1, 64, [40, 7], [4000, 2]
    q = normal(g, 60, H, dim, std=2.0, dtype=BF16)
    k, v = normal(g, 4010, KV, dim, dtype=BF16), normal(g, 4010, KV, dim, dtype=BF16)
    want = reference(q[:47], k[:4002], v[:4002], each, keys, 0, 0, dim ** -0.5)
    k[4002:], v[4002:] = what, what
    v[3980, 0, 5] = what
    k_offsets = ints(starts(keys))
    y, kept = lib.attend_rows(q, k, v, ints(starts(each)), k_offsets=k_offsets, keep=True)
    assert lib.moe_attend_rows_bytes(60, 4010, 2, H, KV, dim) > 0
    assert not y[47:].any() and not y[40:45].any() and bool((kept.lse[:, 40:45] == -math.inf).all())
    sees = torch.arange(40, device=DEV) >= 20
    one = y[:40][sees][:, :, 5].float()
    assert bool((one.isnan() if what != what else one == what).all())
    clean = torch.ones(47, H, dim, dtype=torch.bool, device=DEV)
    clean[:40][sees, :, 5] = False
    over = (y[:47].double() - want["y"][0]).abs() - want["y"][1] * (1 + 2 * U)
    assert float(torch.where(clean, over, -1.0).max()) <= 0


def test_shares_of_keys_with_nan(lib):
    """A NaN that a query has or sees is in its y and lse, whichever share of the keys it is in, as it is without shares; the other
    queries and heads have their values."""
    g = gen(22)
    H, KV, dim, nq, nk = 4, 2, 64, 100, 3900
    q = normal(g, nq, H, dim, std=2.0, dtype=BF16)
    k, v = normal(g, nk, KV, dim, dtype=BF16), normal(g, nk, KV, dim, dtype=BF16)
    assert lib.moe_attend_rows_bytes(nq, nk, 1, H, KV, dim) > 0
    offsets, k_offsets = ints([0, nq]), ints([0, nk])

    def check(q, k, v, bad):
        """bad [nq, H]: what has to be NaN"""
        y, kept = lib.attend_rows(q, k, v, offsets, k_offsets=k_offsets, keep=True)
        assert bool(y.isnan().all(2)[bad].all()) and bool(kept.lse.isnan().t()[bad].all())
        over = (y.double() - want[0]).abs() - want[1] * (1 + 2 * U)
        assert float(over[~bad].max()) <= 0 if bool((~bad).any()) else True
        assert bool(torch.isfinite(kept.lse.t()[~bad]).all())
        # without shares: the same sequence among empty ones, so that there are few keys for each
        empty = [0] * 9
        y, kept = lib.attend_rows(q, k, v, ints(empty + [0, nq]), k_offsets=ints(empty + [0, nk]), keep=True)
        assert lib.moe_attend_rows_bytes(nq, nk, 10, H, KV, dim) == 0
        assert bool(y.isnan().all(2)[bad].all()) and bool(kept.lse.isnan().t()[bad].all()) and bool(torch.isfinite(kept.lse.t()[~bad]).all())

    want = reference(q, k, v, [nq], [nk], 0, 0, dim ** -0.5)["y"]
    none = torch.zeros(nq, H, dtype=torch.bool, device=DEV)
    check(q, k, v, none)
    for rows, value in (((0,), math.nan), ((17, 63, 99), math.nan), (range(nq), math.nan)):  # in queries: in one value, in all of them
        for dims in (slice(5, 6), slice(None)):
            bad, x = none.clone(), q.clone()
            for r in rows:
                bad[r, 1] = True
                x[r, 1, dims] = value
            check(x, k, v, bad)
    bad, x = none.clone(), k.clone()
    bad[:, 2:], x[:, 1, 7] = True, math.nan  # in all keys of a head
    check(q, x, v, bad)
    for tile in range(0, nk // 64 - 6):  # in all keys of tiles, of every share's among them; all queries see them
        for n in (1, 4, 5):
            x = k.clone()
            x[64 * tile:64 * (tile + n), 1, 7] = math.nan
            y, kept = lib.attend_rows(q, x, v, offsets, k_offsets=k_offsets, keep=True)
            assert bool(y[:, 2:].isnan().all()) and bool(kept.lse[2:].isnan().all()) and bool(torch.isfinite(y[:, :2]).all()), (tile, n)


@pytest.mark.parametrize("heads", [2, 48])
def test_nan_in_queries(lib, heads):
    """In every form without shares, and over pages by one workgroup and in shares: NaN for these queries and heads, values for the others."""
    g = gen(25)
    n, dim = 400, 64
    q, k, v = normal(g, n, heads, dim, std=2.0, dtype=BF16), normal(g, n, 1, dim, dtype=BF16), normal(g, n, 1, dim, dtype=BF16)
    want, bound = reference(q, k, v, [n], [n], 0, 0, 0.125)["y"]
    bad = torch.zeros(n, heads, dtype=torch.bool, device=DEV)
    for r in (0, 31, 130, 399):
        q[r, 1, r % dim] = math.nan
        bad[r, 1] = True
    y, kept = lib.attend_rows(q, k, v, ints([0, n]), keep=True)
    assert torch.equal(y.isnan(), bad[..., None].expand_as(y)) and torch.equal(kept.lse.isnan().t(), bad)
    close(y[~bad], want[~bad], bound[~bad], "y")
    for lengths in ([300], [3000, 40]):
        values, pages, _, table = paged(g, lengths, 1, dim, 16, BF16)
        one = normal(g, len(lengths), heads, dim, dtype=BF16)
        want, bound = paged_reference(one, values, 0, 0, 0.125)
        one[0, 1, 5] = math.nan
        y = lib.attend_pages(one, *pages, table, ints(lengths))
        assert bool(y[0, 1].isnan().all()) and int(y.isnan().sum()) == dim
        fine = torch.isfinite(y)
        close(y[fine], want[fine], bound[fine], "pages")


@pytest.mark.parametrize("dim", [64, 80, 128])
@pytest.mark.parametrize("each,keys,heads", [
    ([400], None, 2), ([400], None, 48),  # the keys divided among wavefronts; whole tiles by a workgroup
    ([70], [4000], 2)])                   # shares of the keys
@pytest.mark.parametrize("first,n", [(0, 32), (0, 64), (0, 130), (37, 64), (128, 64), (0, 300)])
def test_scores_of_minus_infinity(lib, dim, each, keys, heads, first, n):
    """Keys that score -infinity with every query weigh nothing, also where a query sees a whole tile of them ahead of any other."""
    g = gen(dim + n)
    nk = sum(keys or each)
    q = normal(g, sum(each), heads, dim, std=2.0, dtype=BF16)
    k, v = (normal(g, nk, 1, dim, dtype=BF16) for _ in range(2))
    q[:, :, 3] = 1.0
    ok = visible(sum(each), nk, 0, 0)
    ok[:, first:first + n] = False
    kept = k.clone()
    k[first:first + n, :, 3] = -math.inf
    y, keep = lib.attend_rows(q, k, v, ints(starts(each)), k_offsets=ints(starts(keys or each)), keep=True)
    some = ok.any(1)
    for h in range(0, heads, max(1, heads // 3)):
        want, bound = one_head(q[:, h].double(), kept[:, 0].double(), v[:, 0].double(), ok, dim ** -0.5)["y"]
        close(y[some, h], want[some], bound[some], (h, "y"))
    assert bool(torch.isfinite(keep.lse[:, some]).all())


@pytest.mark.parametrize("each,keys,heads", [([200], None, 2), ([200], None, 100), ([30], [3000], 2)])
def test_all_scores_minus_infinity(lib, each, keys, heads):
    """As if nothing were seen: zeros and lse -infinity, in every form, over pages, too."""
    g = gen(24)
    nq, nk, dim = sum(each), sum(keys or each), 64
    q, k, v = normal(g, nq, heads, dim, dtype=BF16), normal(g, nk, 1, dim, dtype=BF16), normal(g, nk, 1, dim, dtype=BF16)
    q[:, 0, 3] = 1.0
    k[:, :, 3] = -math.inf
    q[:, 1:, 3] = 2.0
    y, kept = lib.attend_rows(q, k, v, ints(starts(each)), k_offsets=ints(starts(keys or each)), keep=True)
    assert not y.any() and bool((kept.lse == -math.inf).all())
    n = 2900 if keys else 200  # (in shares, and by one workgroup)
    pages = [torch.zeros(up(nk, 16) * 16, 1, dim, dtype=BF16, device=DEV) for _ in range(2)]
    pages[0][:nk], pages[1][:nk] = k, v
    pages = [p.view(-1, 16, 1, dim).transpose(1, 2).contiguous() for p in pages]
    table = torch.arange(pages[0].shape[0], dtype=I32, device=DEV)[None]
    assert not lib.attend_pages(q[:1], *pages, table, ints([n])).any()


def test_gradients_of_other_sequences(lib):
    """An infinity or NaN stays in its sequence's gradients."""
    g = gen(7)
    each = [100, 70, 130]
    offsets = ints(starts(each))
    q, k, v, dy = (normal(g, 310, h, 96, dtype=BF16) for h in (4, 2, 2, 4))
    want = reference(q[:300], k[:300], v[:300], each, each, 0, 0, 96 ** -0.5, dy[:300])
    for t in (q, k, v, dy):
        t[100:170] = math.nan
        t[300:] = math.inf
    y, kept = lib.attend_rows(q, k, v, offsets, keep=True)
    for n, got in zip(("y", "dq", "dk", "dv"), (y, *lib.attend_rows_backward(q, k, v, offsets, y, kept, dy))):
        assert not got[300:].any() and bool(got[100:170].isnan().all())
        rows = torch.tensor([i for i in range(300) if not 100 <= i < 170], device=DEV)
        close(got[rows], want[n][0][rows], want[n][1][rows], n)


def test_offsets_that_do_not_fit(lib):
    """Rows ahead of the first sequence and behind the last; offsets beyond the rows or out of order read nothing out of range."""
    g = gen(3)
    q, k, v, dy = (normal(g, 200, h, 64, dtype=BF16) for h in (2, 1, 1, 2))
    want = reference(q[20:150], k[20:150], v[20:150], [60, 70], [60, 70], 0, 0, 0.125, dy[20:150])
    offsets = ints([20, 80, 150])
    y, kept = lib.attend_rows(q, k, v, offsets, keep=True)
    for n, got in zip(("y", "dq", "dk", "dv"), (y, *lib.attend_rows_backward(q, k, v, offsets, y, kept, dy))):
        assert not got[:20].any() and not got[150:].any()
        close(got[20:150], *want[n], n)
    y = lib.attend_rows(q, k, v, ints([20, 80, 1 << 30]))  # (the last sequence has the rows that there are)
    want = reference(q[20:], k[20:], v[20:], [60, 120], [60, 120], 0, 0, 0.125)
    close(y[20:], *want["y"], "y")
    for bad in ([150, 20, -5], [-(1 << 31), (1 << 31) - 1, 0], [0, 200] * 400, [(7919 * i) % 300 - 50 for i in range(500)]):
        y, kept = lib.attend_rows(q, k, v, ints(bad), keep=True)
        lib.attend_rows_backward(q, k, v, ints(bad), torch.zeros_like(y), lib.KeptAttention(torch.zeros_like(kept.lse), None), dy)
        torch.cuda.synchronize()


def test_ends_of_sequences_far_below_zero(lib):
    """An end so far ahead of its start that their difference passes 32 bits is of a sequence without rows: nothing out of range is read,
    and its neighbours have their rows."""
    least = -(1 << 31)
    g = gen(4)
    q, k, v, dy = (normal(g, 200, h, 64, dtype=BF16) for h in (2, 1, 1, 2))
    for bad in ([150, least, 20], [200, least + 1, -5], [1, least] + [0] * 200, [199, least] * 100, [least, least, 150]):
        for of in (dict(), dict(k_offsets=ints([0] + [200] * (len(bad) - 1)))):
            y, kept = lib.attend_rows(q, k, v, ints(bad), keep=True, **of)
            lib.attend_rows_backward(q, k, v, ints(bad), torch.zeros_like(y), lib.KeptAttention(torch.zeros_like(kept.lse), None), dy, **of)
            torch.cuda.synchronize()
    # keys that end far below zero: their queries see none, the next sequence has its own
    want = reference(q[60:], k[:140], v[:140], [140], [140], 0, 0, 0.125, dy[60:])
    kw = dict(k_offsets=ints([150, least, 140]))
    offsets = ints([0, 60, 200])
    y, kept = lib.attend_rows(q, k, v, offsets, keep=True, **kw)
    assert not y[:60].any()
    close(y[60:], *want["y"], "y")
    dq = lib.attend_rows_backward(q, k, v, offsets, y, kept, dy, **kw)[0]
    assert not dq[:60].any()
    close(dq[60:], *want["dq"], "dq")


@pytest.mark.parametrize("layout", ["heads first", "one projection", "wide", "one head"])
def test_layouts(lib, layout):
    g = gen(11)
    T, H, KV, D = 230, 4, 2, 64
    if layout == "heads first":
        q, k, v = (normal(g, h, T, D, dtype=BF16).transpose(0, 1) for h in (H, KV, KV))
    elif layout == "one projection":
        x = normal(g, T, (H + 2 * KV) * D, dtype=BF16)
        q, k, v = x[:, :H * D].view(T, H, D), x[:, H * D:(H + KV) * D].view(T, KV, D), x[:, (H + KV) * D:].view(T, KV, D)
    elif layout == "wide":
        q, k, v = (normal(g, T, h, 3, D + 8, dtype=BF16)[:, :, 1, :D] for h in (H, KV, KV))
    else:
        H = KV = 1
        q, k, v = (normal(g, T, 1, D, dtype=BF16) for _ in range(3))
    dy = normal(g, T, H, D, dtype=BF16)
    offsets, kw = ints([0, 100, T]), dict(window=50, sinks=2, scale=0.2)
    y, kept = lib.attend_rows(q, k, v, offsets, keep=True, **kw)
    want = reference(q, k, v, [100, T - 100], [100, T - 100], 50, 2, 0.2, dy)
    for n, got in zip(("y", "dq", "dk", "dv"), (y, *lib.attend_rows_backward(q, k, v, offsets, y, kept, dy, **kw))):
        close(got, *want[n], n)


def test_one_row_between_heads_that_lie_far_apart(lib):
    """Of one row there is no stride that could be too large."""
    g = gen(12)
    q, k, v = (normal(g, 4, 1 << 16, 64, dtype=BF16)[:, 70:71].transpose(0, 1) for _ in range(3))
    for x in (q, k, v):
        assert x.shape == (1, 4, 64) and x.stride(1) == 1 << 22
    y, kept = lib.attend_rows(q, k, v, ints([0, 1]), keep=True)
    dy = normal(g, 1, 4, 64, dtype=BF16)
    dq, dk, dv = lib.attend_rows_backward(q, k, v, ints([0, 1]), y, kept, dy)
    assert torch.equal(y, v) and torch.equal(dv, dy)
    pages = torch.zeros(1, 4, 16, 64, dtype=BF16, device=DEV)
    lib.store_pages(k, v, ints([3]), pages, pages.clone())
    assert torch.equal(pages[0, :, 3], k[0])
    assert torch.equal(lib.attend_pages(q, pages, pages, ints([[0]]), ints([4]), window=1)[0], k[0])


def test_caches_of_inference_mode(lib):
    """They are written to in that mode, and refused outside it ahead of the launch."""
    g = gen(14)
    k, slots = normal(g, 2, 1, 64, dtype=BF16), ints([1, 5])
    with torch.inference_mode():
        pages = [torch.zeros(1, 1, 16, 64, dtype=BF16, device=DEV) for _ in range(2)]
        table = ints([[-1]])
        lib.store_pages(k, k, slots, *pages)
        lib.plan_pages(ints([0]), ints([1]), table, ints([7]), 16, 1)
    assert torch.equal(pages[0][0, 0, 5], k[1, 0]) and table.item() == 7
    before = [p.clone() for p in pages]
    for call in (lambda: lib.store_pages(k + 1, k, slots, *pages), lambda: lib.plan_pages(ints([0]), ints([1]), table, ints([8]), 16, 1)):
        with pytest.raises(ValueError, match="inference"):
            call()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(before, pages)) and table.item() == 7


def test_gradients_against_differences(lib):
    """The loss <y, w> along a direction of each input: the gradient's product with it against a central difference of the same
    calls.  q, k, v are whole multiples of 2^-6 up to 2 and steps of 2^-4 keep them bf16.  Third derivatives are below 4 along these
    directions in 64 bits (a step of h gives h^2 / 6 of them), and y's roundings of U each are independent in thousands of terms."""
    g = gen(13)
    T, H, KV, D = 96, 2, 1, 32
    q, k, v = ((normal(g, T, h, D) * 16).round().clamp(-64, 64) / 64 for h in (H, KV, KV))
    w = normal(g, T, H, D, dtype=BF16)
    offsets = ints([0, 40, T])

    def loss(q, k, v):
        return float((lib.attend_rows(q.to(BF16), k.to(BF16), v.to(BF16), offsets, window=30, sinks=2).double() * w.double()).sum())

    def exact(q, k, v):
        return float((reference(q, k, v, [40, T - 40], [40, T - 40], 30, 2, D ** -0.5)["y"][0] * w.double()).sum())

    b = [t.to(BF16) for t in (q, k, v)]
    y, kept = lib.attend_rows(*b, offsets, window=30, sinks=2, keep=True)
    grads = lib.attend_rows_backward(*b, offsets, y, kept, w, window=30, sinks=2)
    h = 2.0 ** -4
    noise = 4 * U * float((y.double() * w.double()).square().sum()) ** 0.5 / h  # (four times the spread of two sums of roundings)
    for i, grad in enumerate(grads):
        step = torch.randint(-1, 2, b[i].shape, generator=g, device=DEV).float()
        plus, minus = [list((q, k, v)) for _ in range(2)]
        plus[i], minus[i] = plus[i] + h * step, minus[i] - h * step
        along = float((grad.double() * step.double()).sum())
        curved = abs((exact(*plus) - exact(*minus)) / (2 * h) - float((reference(*b, [40, T - 40], [40, T - 40], 30, 2, D ** -0.5, w)[("dq", "dk", "dv")[i]][0] * step.double()).sum()))
        size = 4 * U * float((grad.double() * step.double()).square().sum()) ** 0.5
        assert abs((loss(*plus) - loss(*minus)) / (2 * h) - along) <= noise + size + curved, i


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
    ([i % 7 * 9 for i in range(1500)] + [2500], 2, 1, 64, 16, 0, 0),
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


@pytest.mark.parametrize("lengths,heads,kv,dim,page,window,sinks", [
    ([1, 2, 40, 700], 4, 2, 128, 16, 0, 0),                   # a workgroup for each
    ([5000, 1, 3, 900, 0, 64], 8, 2, 64, 32, 0, 0),           # in shares
    ([5000, 1, 3, 900, 0, 64], 8, 2, 128, 16, 0, 0),
    ([3000, 1, 500] * 40, 6, 2, 72, 16, 0, 0),                # ... joined by wavefronts
    ([1500, 40, 700], 8, 2, 128, 16, 100, 4)])
def test_infinities_in_pages(lib, lengths, heads, kv, dim, page, window, sinks):
    """An infinity or NaN in a value that is seen is in y's dim of the heads that read it, as it is over rows; in a key, NaN."""
    g = gen(dim + len(lengths))
    values, pages, _, table = paged(g, lengths, kv, dim, page, BF16)
    q = normal(g, len(lengths), heads, dim, std=2.0, dtype=BF16)
    want, bound = paged_reference(q, values, window, sinks, dim ** -0.5)
    expect = want.clone()
    per = heads // kv

    def put(cache, i, pos, head, d, value):
        cache[int(table[i, pos // page]), head, pos % page, d] = value

    for i, n in enumerate(lengths):
        if n == 0:
            continue
        seen = visible(1, n, window, sinks)[0].nonzero()[:, 0].tolist()
        for pos, d, value in ((n - 1, 0, math.inf), (seen[0], 1, -math.inf), (seen[len(seen) // 2], 2, math.nan), (n - 1, 3, math.inf), (seen[0], 3, math.inf),
                              (seen[len(seen) // 3], 4, -math.inf)):
            put(pages[1], i, pos, 0, d, value)
            expect[i, :per, d] = value
        if len(seen) > 1:  # both infinities in one dim
            put(pages[1], i, seen[0], 0, 5, math.inf)
            put(pages[1], i, n - 1, 0, 5, -math.inf)
            expect[i, :per, 5] = math.nan
        if len(seen) < n:  # not seen
            hidden = sorted(set(range(n)) - set(seen))
            put(pages[1], i, hidden[-1], 0, 6, math.inf)
            put(pages[0], i, hidden[len(hidden) // 2], 0, 6, math.nan)
        if i % 2:
            put(pages[0], i, seen[len(seen) // 4], 1, 7, math.nan)
            expect[i, per:2 * per] = math.nan
    y = lib.attend_pages(q, *pages, table, ints(lengths), window=window, sinks=sinks).double()
    assert torch.equal(y.isnan(), expect.isnan())
    odd = expect.isinf()
    assert torch.equal(y.isinf(), odd) and torch.equal(y[odd], expect[odd])
    fine = torch.isfinite(expect)
    close(y[fine], want[fine], bound[fine], "y")


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


@pytest.mark.parametrize("cache", [BF16, I8])
@pytest.mark.parametrize("window,sinks", [(0, 0), ((1 << 31) - 1, 0), ((1 << 30) + 5000, 0), ((1 << 30) + 5000, 700), (50, (1 << 30) + 100), (300, 5), (1 << 30, 1 << 30)])
def test_as_many_tokens_as_lengths_count(lib, cache, window, sinks):
    """2^31 - 1 of them, of which few pages are there: positions, windows and first keys that pass 2^30, and the last token of all."""
    page, n, dim = 1024, (1 << 31) - 1, 64
    entries = [0, 1, (1 << 20) - 5, 1 << 20, (1 << 21) - 2, (1 << 21) - 1]
    g = gen(41)
    values, pages, scales, few = paged(g, [len(entries) * page - 1], 1, dim, page, cache)
    table = torch.full((1, 1 << 21), -1, dtype=I32, device=DEV)
    table[0, entries] = few[0, :len(entries)]
    q = normal(g, 1, 2, dim, std=2.0, dtype=BF16)
    pos = (torch.tensor(entries, device=DEV)[:, None] * page + torch.arange(page, device=DEV)).reshape(-1)[:-1]
    assert int(pos[-1]) == n - 1
    seen = torch.ones_like(pos, dtype=torch.bool) if window == 0 else (pos > n - 1 - window) | (pos < sinks)
    want = paged_reference(q, [[x[seen] for x in values[0]]], 0, 0, dim ** -0.5)
    close(lib.attend_pages(q, *pages, table, ints([n]), *scales, window=window, sinks=sinks), *want, "y")


# ---- how the calls are made --------------------------------------------------------------------------------
def serve_setup(lib, cache=BF16, seed=17, **kw):
    """Three requests: their prompts by attend_rows, stored; then tokens one by one."""
    g = gen(seed)
    H, KV, D, page, prompts, steps = 4, 2, 64, 16, [37, 1, 90], 20
    n = [p + steps for p in prompts]
    q = [normal(g, m, H, D, std=2.0, dtype=BF16) for m in n]
    k, v = ([normal(g, m, KV, D, dtype=BF16) for m in n] for _ in range(2))
    pages = [torch.full((40, KV, page, D), math.nan, device=DEV).to(BF16) if cache == BF16 else torch.full((40, KV, page, D), 3, dtype=I8, device=DEV) for _ in range(2)]
    scales = [torch.full((40, KV, page), math.nan, device=DEV) for _ in range(2)] if cache == I8 else [None, None]
    return dict(H=H, KV=KV, D=D, page=page, prompts=prompts, steps=steps, q=q, k=k, v=v, pages=pages, scales=scales, table=torch.full((3, 8), -1, dtype=I32, device=DEV),
                free=torch.randperm(40, generator=g, device=DEV).int())


def step_rows(s, key, t):
    return torch.stack([x[p + t] for x, p in zip(s[key], s["prompts"])])


@pytest.mark.parametrize("cache", [BF16, I8])
@pytest.mark.parametrize("window,sinks", [(0, 0), (24, 3)])
def test_prompts_then_tokens(lib, cache, window, sinks):
    """plan, store and both attentions together: tokens one by one give what the whole sequence gives at once."""
    s = serve_setup(lib, cache)
    want = []
    for q, k, v in zip(s["q"], s["k"], s["v"]):
        want.append(reference(q, k, v, [q.shape[0]], [q.shape[0]], window, sinks, s["D"] ** -0.5)["y"])
    cat = lambda key: torch.cat([x[:p] for x, p in zip(s[key], s["prompts"])])  # noqa: E731
    plan = lib.plan_pages(ints([0, 0, 0]), ints(s["prompts"]), s["table"], s["free"], s["page"], sum(s["prompts"]) + 3)
    pad = torch.nn.functional.pad
    rows = [pad(cat(key), (0, 0, 0, 0, 0, 3)) for key in ("q", "k", "v")]
    y = lib.attend_rows(*rows, plan.offsets, window=window, sinks=sinks)
    assert not y[-3:].any()
    for i, p in enumerate(s["prompts"]):
        a = int(plan.offsets[i])
        close(y[a:a + p], want[i][0][:p], want[i][1][:p], "prompt")
    lib.store_pages(rows[1], rows[2], plan.slots, *s["pages"], *s["scales"])
    ones = ints([1, 1, 1])
    for t in range(s["steps"]):
        plan = lib.plan_pages(plan.lengths, ones, s["table"], s["free"], s["page"], 3, used=plan.used)
        lib.store_pages(step_rows(s, "k", t), step_rows(s, "v", t), plan.slots, *s["pages"], *s["scales"])
        y = lib.attend_pages(step_rows(s, "q", t), *s["pages"], s["table"], plan.lengths, *s["scales"], window=window, sinks=sinks)
        for i, p in enumerate(s["prompts"]):
            if cache == BF16:
                close(y[i], want[i][0][p + t], want[i][1][p + t], "token")
            else:  # a code is off by half a step of 1/127 of the largest of 64 normal values (2.5) at most, at random in each key and value
                assert float((y[i].double() - want[i][0][p + t]).norm() / want[i][0][p + t].norm()) <= 0.05
    assert plan.lengths.tolist() == [p + s["steps"] for p in s["prompts"]]
    assert int(plan.used) == sum(up(p + s["steps"], s["page"]) for p in s["prompts"])


def test_a_captured_step_is_replayed(lib):
    """One decoding step as a graph: plan, store, attend; lengths and used go round in the graph's own tensors."""
    s = serve_setup(lib)
    pad_rows = [torch.cat([x[:p] for x, p in zip(s[key], s["prompts"])]) for key in ("k", "v")]
    first = lib.plan_pages(ints([0, 0, 0]), ints(s["prompts"]), s["table"], s["free"], s["page"], sum(s["prompts"]))
    lib.store_pages(*pad_rows, first.slots, *s["pages"])
    have, used, ones = first.lengths.clone(), first.used.clone(), ints([1, 1, 1])
    q, k, v = (step_rows(s, key, 0).clone() for key in ("q", "k", "v"))

    def step():
        plan = lib.plan_pages(have, ones, s["table"], s["free"], s["page"], 3, used=used)
        lib.store_pages(k, v, plan.slots, *s["pages"])
        y = lib.attend_pages(q, *s["pages"], s["table"], plan.lengths)
        have.copy_(plan.lengths)
        used.copy_(plan.used)
        return y

    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        out = step()
    other = torch.randn(1 << 20, device=DEV)
    for t in range(s["steps"]):
        for to, key in ((q, "q"), (k, "k"), (v, "v")):
            to.copy_(step_rows(s, key, t))
        graph.replay()
        other = other * 1.5 - other.mean()  # (the program's own work in between)
        if t % 3 == 0:
            torch.cuda.synchronize()
        for i, p in enumerate(s["prompts"]):
            n = p + t + 1
            want = reference(s["q"][i][:n], s["k"][i][:n], s["v"][i][:n], [n], [n], 0, 0, s["D"] ** -0.5)["y"]
            close(out[i], want[0][-1], want[1][-1], (t, i))


@pytest.mark.parametrize("each,keys,heads", [([300, 1000], [300, 1000], 16), ([30, 100], [1700, 2000], 2)])
def test_captured_gradients_beside_eager_ones(lib, each, keys, heads):
    """attend_rows and its backward in a graph, replayed on other inputs, with eager calls of the same kind in between."""
    g = gen(23)
    offsets, k_offsets = ints(starts(each)), ints(starts(keys))
    ts = [normal(g, n, h, 64, dtype=BF16) for n, h in ((sum(each), heads), (sum(keys), 1), (sum(keys), 1), (sum(each), heads))]

    def both(q, k, v, dy):
        y, kept = lib.attend_rows(q, k, v, offsets, k_offsets=k_offsets, keep=True)
        return (y, *lib.attend_rows_backward(q, k, v, offsets, y, kept, dy, k_offsets=k_offsets))

    both(*ts)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        out = both(*ts)
    for seed in range(4):
        new = [normal(gen(100 + seed), *t.shape, dtype=BF16) for t in ts]
        for t, n in zip(ts, new):
            t.copy_(n)
        graph.replay()
        eager = both(*new)
        torch.cuda.synchronize()
        for a, b in zip(out, eager):
            assert torch.equal(a, b)


def test_streams_and_calls_at_once(lib):
    """The calls go to the current stream; two at once have workspaces of their own."""
    g = gen(29)
    values, pages, _, table = paged(g, [3000, 40, 900], 2, 128, 16, BF16)
    q = normal(g, 3, 8, 128, dtype=BF16)
    want = paged_reference(q, values, 0, 0, 128 ** -0.5)
    lengths = ints([3000, 40, 900])
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(3)]
    out = []
    for _ in range(4):
        for s in streams:
            with torch.cuda.stream(s):
                out.append(lib.attend_pages(q, *pages, table, lengths))
    torch.cuda.synchronize()
    close(out[0], *want, "y")
    assert all(torch.equal(out[0], y) for y in out)


def test_calls_at_once_of_different_work(lib):
    """Calls on three streams, each with lengths, queries and rows of its own and so with other shares, pieces and parts in its workspace:
    over pages, over rows with their keys in shares, and gradients in pieces and shares."""
    jobs = []
    for i, (lengths, each, keys, each2) in enumerate((([3000, 40, 900], [60, 9], [2500, 1900], [700, 41]), ([17, 5000], [100], [4000], [900]),
                                                      ([2100, 1, 1300, 60], [5, 33, 20], [1800, 2000, 1700], [300, 300, 333]))):
        g = gen(60 + i)
        values, pages, _, table = paged(g, lengths, 2, 128, 16, BF16)
        q = normal(g, len(lengths), 8, 128, dtype=BF16)
        qr, k, v = normal(g, sum(each), 2, 64, dtype=BF16), normal(g, sum(keys), 1, 64, dtype=BF16), normal(g, sum(keys), 1, 64, dtype=BF16)
        q2, k2, v2, dy2 = (normal(g, sum(each2), h, 64, dtype=BF16) for h in (8, 1, 1, 8))
        offsets, k_offsets, offsets2, n = ints(starts(each)), ints(starts(keys)), ints(starts(each2)), ints(lengths)
        assert lib.moe_attend_rows_bytes(sum(each), sum(keys), len(each), 2, 1, 64) > 0
        want = (paged_reference(q, values, 0, 0, 128 ** -0.5), reference(qr, k, v, each, keys, 0, 0, 0.125)["y"],
                *(reference(q2, k2, v2, each2, each2, 0, 0, 0.125, dy2)[x] for x in ("y", "dq", "dk", "dv")))

        def run(q=q, pages=pages, table=table, n=n, rows=(qr, k, v, offsets), k_offsets=k_offsets, rows2=(q2, k2, v2, offsets2), dy2=dy2):
            y = lib.attend_pages(q, *pages, table, n)
            y1 = lib.attend_rows(*rows, k_offsets=k_offsets)
            y2, kept = lib.attend_rows(*rows2, keep=True)
            return (y, y1, y2, *lib.attend_rows_backward(*rows2, y2, kept, dy2))

        jobs.append((torch.cuda.Stream(), run, want, []))
    torch.cuda.synchronize()
    for _ in range(6):
        for stream, run, _, out in jobs:
            with torch.cuda.stream(stream):
                out.append(run())
    torch.cuda.synchronize()
    for _, _, want, out in jobs:
        for got, (ref, bound), what in zip(out[0], want, ("pages", "shares", "y", "dq", "dk", "dv")):
            close(got, ref, bound, what)
        for other in out[1:]:
            assert all(torch.equal(a, b) for a, b in zip(out[0], other))


def test_offsets_in_a_large_cache(lib):
    """Pages beyond 2^32 bytes of the cache."""
    KV, page, D = 8, 64, 128
    n = (1 << 32) // (KV * page * D * 2) + 40
    pages = [torch.empty(n, KV, page, D, dtype=BF16, device=DEV) for _ in range(2)]
    g = gen(31)
    ids = torch.tensor([n - 1, 3, n - 7, (1 << 32) // (KV * page * D * 2)], dtype=I32, device=DEV)
    k, v = (normal(g, 250, KV, D, dtype=BF16) for _ in range(2))
    pos = torch.arange(250, device=DEV)
    lib.store_pages(k, v, (ids[pos // page] * page + pos % page).int(), *pages)
    for x, p in zip((k, v), pages):
        assert torch.equal(p[ids.long()].transpose(1, 2).reshape(-1, KV, D)[:250], x)
    q = normal(g, 1, 16, D, std=2.0, dtype=BF16)
    y = lib.attend_pages(q, *pages, ids[None].contiguous(), ints([250]))
    close(y, *paged_reference(q, [[k.double(), v.double()]], 0, 0, D ** -0.5), "y")


def test_nothing_to_do(lib):
    empty = torch.empty(0, 4, 64, dtype=BF16, device=DEV)
    y, kept = lib.attend_rows(empty, empty[:, :2], empty[:, :2], ints([0]), keep=True)
    assert y.shape == empty.shape and kept.lse.shape == (4, 0)
    k = torch.randn(10, 2, 64, device=DEV).to(BF16)
    y, kept = lib.attend_rows(empty, k, k, ints([0, 0]), k_offsets=ints([0, 10]), keep=True)
    dq, dk, dv = lib.attend_rows_backward(empty, k, k, ints([0, 0]), y, kept, empty, k_offsets=ints([0, 10]))
    assert dq.shape == empty.shape and not dk.any() and not dv.any()
    q = torch.randn(10, 4, 64, device=DEV).to(BF16)
    none = torch.empty(0, 2, 64, dtype=BF16, device=DEV)
    y = lib.attend_rows(q, none, none, ints([0, 10]), k_offsets=ints([0, 0]))
    assert not y.any()
    y = lib.attend_rows(q, k, k, ints([0]))  # (no sequence)
    assert not y.any()
    pages = torch.empty(0, 2, 16, 64, dtype=BF16, device=DEV)
    y = lib.attend_pages(q, pages, pages, torch.zeros(10, 3, dtype=I32, device=DEV), ints([5] * 10))
    assert not y.any()
    lib.store_pages(k, k, ints([0] * 10), pages, pages)
    assert lib.attend_pages(empty, pages, pages, torch.zeros(0, 3, dtype=I32, device=DEV), ints([])).shape == empty.shape


def test_gradients_are_not_lost_silently(lib):
    q = torch.randn(10, 2, 64, device=DEV).to(BF16).requires_grad_()
    with pytest.raises(ValueError, match="gradient"):
        lib.attend_rows(q, q, q, ints([0, 10]))
    with torch.no_grad():
        lib.attend_rows(q, q, q, ints([0, 10]))


def test_sizes_are_refused_before_memory_is_taken(lib):
    q = torch.zeros(1024, 1, 512, dtype=BF16, device=DEV).expand(1024, 600, 512)
    torch.cuda.synchronize()
    torch.cuda.reset_peak_memory_stats()
    before = torch.cuda.memory_allocated()
    with pytest.raises((lib.MoEError, ValueError)):
        lib.attend_rows(q, q, q, ints([0, 1024]), keep=True)
    with pytest.raises((lib.MoEError, ValueError)):
        lib.plan_pages(ints([1]), ints([1]), ints([[0]]), ints([1]), 16, 1 << 30)
    assert torch.cuda.max_memory_allocated() - before < 1 << 16


def test_calls_through_the_c_entry_points(lib):
    """Without tensors' part: pointers, another stream, a cache written in place."""
    g = gen(37)
    q, k, v = normal(g, 70, 2, 64, dtype=BF16), normal(g, 70, 2, 64, dtype=BF16), normal(g, 70, 2, 64, dtype=BF16)
    offsets, y = ints([0, 70]), torch.full((70, 2, 64), 9.0, device=DEV).to(BF16)
    stream = torch.cuda.Stream()
    torch.cuda.synchronize()
    P = lambda t: None if t is None else t.data_ptr()  # noqa: E731
    lib.moe_attend_rows(P(q), 128, 64, P(k), 128, 64, P(v), 128, 64, P(offsets), None, 1, 70, 70, 2, 2, 64, 0.125, 0, 0, P(y), None, None, None, 0, stream.cuda_stream)
    stream.synchronize()
    close(y, *reference(q, k, v, [70], [70], 0, 0, 0.125)["y"], "y")
    assert torch.equal(y, lib.attend_rows(q, k, v, offsets))
