"""The operators on many rows against plain implementations in 64 bits.

Bounds are derived from the number formats: u32 = 2^-24 and u16 = 2^-8 are the largest relative errors of one rounding to
fp32 and bf16.  A sum of n terms in 32 bits, in whatever order, is within n u32 of the sum of the terms' sizes; the kernels' sums
are trees over lanes and short chains, far shorter than n, so 64 u32 holds for every length here.
"""
import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U32, U16 = 2.0 ** -24, 2.0 ** -8
F32, BF16, I8 = torch.float32, torch.bfloat16, torch.int8


def gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def normal(g, *shape, dtype=F32, std=1.0):
    return (torch.randn(*shape, generator=g, device=DEV) * std).to(dtype)


def unit(dtype):
    return U32 if dtype == F32 else U16


def within(got, ref, bound, what=""):
    off = (got.double() - ref).abs()
    assert bool((off <= bound).all()), (what, float(off.max()), float((off - bound).max()))


# ---- norm -------------------------------------------------------------------------------------------------------
WIDTHS = [1, 63, 64, 100, 513, 1001, 1024, 2048, 2050, 4096, 5000, 8191, 8192]


@pytest.mark.parametrize("hidden", WIDTHS)
@pytest.mark.parametrize("rows", [1, 5, 1500])
@pytest.mark.parametrize("ht,yt", [(F32, BF16), (BF16, F32), (F32, None), (BF16, BF16)])
def test_norm(lib, hidden, rows, ht, yt):
    g = gen(hidden + rows)
    h = normal(g, rows, hidden, dtype=ht, std=3.0)
    y = normal(g, rows, hidden, dtype=yt) if yt else None
    gain = 1 + normal(g, hidden, std=0.2)
    total = h if y is None else (h.float() + y.float()).to(ht)
    s = total.double()
    rstd = (s.square().mean(1, keepdim=True) + 1e-6).rsqrt()
    for out in (F32, BF16, I8):
        n = lib.norm_rows(h, y, gain, out=out)
        assert torch.equal(n.h, total)
        within(n.rstd, rstd[:, 0], 64 * U32 * rstd[:, 0], "rstd")
        if out != I8:
            x = s * rstd * gain.double()
            within(n.x, x, x.abs() * (64 * U32 + (0 if out == F32 else U16)), "x")
            continue
        # the codes are decided by four single-rounding steps
        v = total.float() * gain
        top = v.abs().amax(1, keepdim=True)
        # (in a row of zeros, which a width of one has now and then, the steps are 0 * inf: codes of 0)
        assert torch.equal(n.x.float(), torch.where(top > 0, torch.round(v * (127.0 / top)), 0.0))
        assert int(n.x.abs().max()) == 127
        within(n.scale, (top.double() / 127 * rstd)[:, 0], 64 * U32 * (top.double() / 127 * rstd)[:, 0], "scale")


def test_norm_without_gain_with_strides_and_in_place(lib):
    g = gen(3)
    wide_h, wide_y = normal(g, 33, 1200), normal(g, 33, 999, dtype=BF16)
    for d, off in ((1024, 8), (1024, 1), (700, 3)):
        if d > 990:
            y = wide_y[:, off:off + 990]
            h = wide_h[:, off:off + 990]
        else:
            y, h = wide_y[:, off:off + d], wide_h[:, off:off + d]
        n = lib.norm_rows(h, y, out=F32)
        total = h + y.float()
        assert torch.equal(n.h, total)
        x = total.double() * (total.double().square().mean(1, keepdim=True) + 1e-6).rsqrt()
        within(n.x, x, 64 * U32 * x.abs())
    # the sum may overwrite h (the C entry point)
    from paper_2412_00099_amd import binding as B
    h, y = normal(g, 9, 512), normal(g, 9, 512)
    ref = lib.norm_rows(h, y, out=BF16)
    x = torch.empty(9, 512, dtype=BF16, device=DEV)
    B.moe_norm_rows(h.data_ptr(), B.MOE_R_FP32, 512, y.data_ptr(), B.MOE_R_FP32, 512, None, 1e-6, 9, 512, h.data_ptr(), x.data_ptr(),
                    B.MOE_R_BF16, None, None, torch.cuda.current_stream().cuda_stream)
    assert torch.equal(h, ref.h) and torch.equal(x, ref.x)


def test_norm_of_zeros_and_of_what_is_not_a_number(lib):
    for d in (512, 77):
        h = normal(gen(5), 6, d)
        h[1] = 0
        h[2, 3] = float("inf")
        h[3, 5] = float("nan")
        h[4] = 1e-35
        clean = lib.norm_rows(normal(gen(5), 6, d), out=I8)
        n = lib.norm_rows(h, out=I8)
        for r in (0, 5):
            assert torch.equal(n.x[r], clean.x[r]) and n.scale[r] == clean.scale[r]
        for r in (1, 4):
            assert not n.x[r].any() and n.scale[r] == 0
        for r in (2, 3):
            assert not n.x[r].any() and torch.isnan(n.scale[r])
        x = lib.norm_rows(h, out=F32).x
        assert not x[1].any() and torch.isnan(x[2, 3]) and torch.isnan(x[3]).all() and torch.isfinite(x[5]).all()


def test_norm_empty(lib):
    n = lib.norm_rows(torch.empty(0, 64, device=DEV), gain=torch.ones(64, device=DEV), out=I8)
    assert n.x.shape == (0, 64)
    dh, dgain = lib.norm_rows_backward(n.h, torch.ones(64, device=DEV), n.rstd, torch.empty(0, 64, device=DEV))
    assert dh.shape == (0, 64) and not dgain.any()


@pytest.mark.parametrize("hidden", [1, 100, 513, 1024, 2048, 3001, 8191, 8192])
@pytest.mark.parametrize("rows", [1, 7, 1100])
@pytest.mark.parametrize("ht,xt", [(F32, BF16), (BF16, F32), (F32, F32), (BF16, BF16)])
def test_norm_backward(lib, hidden, rows, ht, xt):
    g = gen(7 * hidden + rows)
    h, gain = normal(g, rows, hidden, dtype=ht, std=2.0), 1 + normal(g, hidden, std=0.2)
    dx, up = normal(g, rows, hidden, dtype=xt), normal(g, rows, hidden, dtype=ht)
    rstd = lib.norm_rows(h, gain=gain).rstd
    n = h.double() * (h.double().square().mean(1, keepdim=True) + 1e-6).rsqrt()
    r = rstd.double()[:, None]
    gx = dx.double() * gain.double()
    own = r * (gx - n * (gx * n).mean(1, keepdim=True))
    size = r * (gx.abs() + n.abs() * (gx * n).abs().mean(1, keepdim=True))
    for d_up in (up, None):
        dh, dgain = lib.norm_rows_backward(h, gain, rstd, dx, d_up)
        ref = own if d_up is None else own + up.double()
        within(dh, ref, 128 * U32 * (size + ref.abs()) + (0 if ht == F32 else U16 * ref.abs()), "dh")
        within(dgain, (dx.double() * n).sum(0), 128 * U32 * (dx.double() * n).abs().sum(0), "dgain")
    assert lib.norm_rows_backward(h, None, rstd, dx)[1] is None
    again = lib.norm_rows_backward(h, gain, rstd, dx, up)
    assert torch.equal(again[1], dgain) or d_up is None
    assert torch.equal(lib.norm_rows_backward(h, gain, rstd, dx, up)[0], again[0])


def test_norm_backward_against_differences(lib):
    """<gradient, direction> against the central difference of the 64-bit function."""
    g = gen(11)
    h, gain, dx = normal(g, 3, 200, std=2.0), 1 + normal(g, 200, std=0.2), normal(g, 3, 200)
    dh, dgain = lib.norm_rows_backward(h, gain, lib.norm_rows(h, gain=gain, out=F32).rstd, dx)

    def f(hh, gg):
        return (dx.double() * hh * (hh.square().mean(1, keepdim=True) + 1e-6).rsqrt() * gg).sum()

    for v, grad, at in ((normal(g, 3, 200).double(), dh, 0), (normal(g, 200).double(), dgain, 1)):
        args = [h.double(), gain.double()]
        e = 1e-4
        hi, lo = list(args), list(args)
        hi[at], lo[at] = args[at] + e * v, args[at] - e * v
        quotient = (f(*hi) - f(*lo)) / (2 * e)
        # (difference: e^2 of a third derivative of order one; gradient: roundings of 600 terms)
        assert abs(float(quotient - (grad.double() * v).sum())) < 1e-5 * float((grad.double() * v).abs().sum()) + 1e-6


# ---- order ------------------------------------------------------------------------------------------------------
def plain_order(ids, n_experts):
    flat = ids.reshape(-1).tolist()
    entry = [p for e in range(n_experts) for p, x in enumerate(flat) if x == e]
    counts = [sum(1 for x in flat if x == e) for e in range(n_experts)]
    offsets = [0]
    for c in counts:
        offsets.append(offsets[-1] + c)
    row = [-1] * len(flat)
    for r, p in enumerate(entry):
        row[p] = r
    return offsets, row, entry + [-1] * (len(flat) - len(entry))


def ids_of(g, tokens, top_k, n_experts, empty):
    ids = torch.rand(tokens, n_experts, generator=g, device=DEV).topk(top_k, 1).indices.int()
    return ids.masked_fill(torch.rand(tokens, top_k, generator=g, device=DEV) < empty, -1).contiguous()


@pytest.mark.parametrize("tokens,top_k,n_experts,empty", [
    (1, 1, 1, 0.0), (1, 8, 8, 0.0), (1, 4, 60, 1.0), (3, 2, 5, 0.4), (64, 1, 64, 0.0), (65, 3, 63, 0.1), (500, 4, 60, 0.0),
    (700, 8, 512, 0.5), (129, 2, 128, 0.0), (300, 8, 127, 0.0)])
def test_sort(lib, tokens, top_k, n_experts, empty):
    ids = ids_of(gen(tokens + n_experts), tokens, top_k, n_experts, empty)
    o = lib.sort_tokens(ids, n_experts)
    offsets, row, entry = plain_order(ids, n_experts)
    assert o.offsets.tolist() == offsets and o.row_of.reshape(-1).tolist() == row and o.entry_of.tolist() == entry


@pytest.mark.parametrize("n_experts", [7, 64, 300])
def test_sort_long(lib, n_experts):
    """Over many workgroups: against a stable library sort; ids that are no experts on both sides of the range."""
    ids = torch.randint(-3, n_experts + 3, (40001, 5), generator=gen(n_experts), device=DEV, dtype=torch.int32)
    ids[:, 2] = 3  # (one expert takes a place of every token)
    o = lib.sort_tokens(ids, n_experts)
    flat = ids.reshape(-1).long()
    inside = (flat >= 0) & (flat < n_experts)
    entry = torch.sort(torch.where(inside, flat, n_experts), stable=True).indices
    n = int(inside.sum())
    assert torch.equal(o.entry_of[:n].long(), entry[:n]) and bool((o.entry_of[n:] == -1).all())
    assert torch.equal(o.offsets.diff().long(), torch.bincount(flat[inside], minlength=n_experts))
    row = torch.full_like(flat, -1)
    row[entry[:n]] = torch.arange(n, device=DEV)
    assert torch.equal(o.row_of.reshape(-1).long(), row)


def test_sort_empty(lib):
    o = lib.sort_tokens(torch.empty(0, 4, dtype=torch.int32, device=DEV), 9)
    assert o.offsets.tolist() == [0] * 10 and o.row_of.shape == (0, 4)


@pytest.mark.parametrize("hidden", [1, 7, 64, 1001, 2048, 8191])
@pytest.mark.parametrize("tokens,top_k,empty", [(1, 1, 0.0), (1, 5, 1.0), (37, 3, 0.3), (200, 8, 0.0), (90, 2, 0.97)])
@pytest.mark.parametrize("dtype,yt", [(F32, F32), (BF16, BF16), (BF16, F32), (F32, BF16)])
def test_rows_there_and_back(lib, hidden, tokens, top_k, empty, dtype, yt):
    g = gen(hidden * tokens + top_k)
    ids = ids_of(g, tokens, top_k, 16, empty)
    o = lib.sort_tokens(ids, 16)
    entry, row = o.entry_of.long(), o.row_of.long()
    there = entry >= 0
    n = int(there.sum())
    x = normal(g, tokens, hidden, dtype=dtype)
    xs, none = lib.gather_rows(x, o)
    assert none is None and torch.equal(xs[:n], x[entry[:n] // top_k]) and not xs[n:].any()
    # whatever lies in rows of nobody, and in weights of empty places, stays out
    ys = normal(g, tokens * top_k, hidden, dtype=dtype)
    ys[n:] = float("nan")
    weight = torch.rand(tokens, top_k, generator=g, device=DEV)
    weight[ids < 0] = float("inf")
    base = normal(g, tokens, hidden, dtype=yt)
    terms = torch.where((row >= 0)[..., None], ys.double()[row.clamp(min=0)] * weight.double()[..., None], 0.0)
    ones = torch.where((row >= 0)[..., None], ys.double()[row.clamp(min=0)], 0.0)
    round_ = 0 if yt == F32 else U16
    for w, t in ((weight, terms), (None, ones)):
        for b in (base, None):
            ref = t.sum(1) + (b.double() if b is not None else 0)
            size = t.abs().sum(1) + (b.double().abs() if b is not None else 0)
            within(lib.combine_rows(ys, o, w, base=b, out=yt), ref, 32 * U32 * size + round_ * ref.abs(), "y")
    dy = normal(g, tokens, hidden, dtype=yt)
    dys, dweight = lib.combine_rows_backward(dy, ys, o, weight)
    ref = dy.double()[entry[:n] // top_k] * weight.double().reshape(-1)[entry[:n], None]
    within(dys[:n], ref, ref.abs() * (2 * U32 if dtype == F32 else U16), "dys")
    assert not dys[n:].any()
    prod = torch.where((row >= 0)[..., None], dy.double()[:, None] * ys.double()[row.clamp(min=0)], 0.0)
    within(dweight, prod.sum(2), 256 * U32 * prod.abs().sum(2), "dweight")
    plain, none = lib.combine_rows_backward(dy, ys, o)
    assert none is None and torch.equal(plain[:n], dy[entry[:n] // top_k].to(dtype))


def test_gather_codes_scales_and_strides(lib):
    g = gen(21)
    ids = ids_of(g, 50, 3, 9, 0.2)
    o = lib.sort_tokens(ids, 9)
    n = int(o.offsets[-1])
    token = o.entry_of.long()[:n] // 3
    wide = torch.randint(-127, 128, (50, 300), generator=g, device=DEV, dtype=torch.int32).to(I8)
    scale = torch.rand(50, generator=g, device=DEV)
    for lo, hi in ((0, 256), (16, 272), (4, 20), (2, 44), (1, 258)):
        xs, ss = lib.gather_rows(wide[:, lo:hi], o, scale=scale)
        assert torch.equal(xs[:n], wide[:, lo:hi][token]) and not xs[n:].any()
        assert torch.equal(ss[:n], scale[token]) and not ss[n:].any()


def test_sum_of_rows_is_the_gradient_of_gather(lib):
    """<gather(v), w> = <v, combine(w)> for every v, w: the two are each other's transpose."""
    g = gen(22)
    o = lib.sort_tokens(ids_of(g, 60, 4, 12, 0.25), 12)
    v, w = normal(g, 60, 96), normal(g, 240, 96)
    a = (lib.gather_rows(v, o)[0].double() * w.double()).sum()
    b = (v.double() * lib.combine_rows(w, o).double()).sum()
    assert abs(float(a - b)) < 1e-6 * float((lib.gather_rows(v, o)[0].double() * w.double()).abs().sum())


def test_combine_backward_against_differences(lib):
    g = gen(23)
    o = lib.sort_tokens(ids_of(g, 10, 3, 6, 0.2), 6)
    ys, weight, dy = normal(g, 30, 40), torch.rand(10, 3, generator=g, device=DEV), normal(g, 10, 40)
    dys, dweight = lib.combine_rows_backward(dy, ys, o, weight)
    row = o.row_of.long()

    def f(a, w):
        rows = torch.where((row >= 0)[..., None], a[row.clamp(min=0)], 0.0)
        return ((rows * w[..., None]).sum(1) * dy.double()).sum()

    a, w = ys.double(), weight.double()
    va, vw = normal(g, 30, 40).double(), normal(g, 10, 3).double()
    e = 1e-3  # (linear in each: the difference is exact up to rounding)
    for quotient, mine in ((f(a + e * va, w) - f(a - e * va, w), dys.double() * va), (f(a, w + e * vw) - f(a, w - e * vw), dweight.double() * vw)):
        assert abs(float(quotient / (2 * e) - mine.sum())) < 1e-5 * float(mine.abs().sum())


# ---- experts ----------------------------------------------------------------------------------------------------
def make_blobs(lib, g, fmt, n, hidden, inter):
    """Packed blobs and the dense weights they stand for, in 64 bits."""
    from paper_2412_00099_amd import binding as B
    f = B.WEIGHT_FMT[fmt]
    blobs = torch.zeros(n, B.moe_blob_bytes(f, hidden, inter), dtype=torch.uint8, device=DEV)
    dense = []
    stream = torch.cuda.current_stream().cuda_stream
    for e in range(n):
        shapes = ((inter, hidden), (inter, hidden), (hidden, inter))
        if fmt == "bf16":
            w = [normal(g, *s, dtype=BF16, std=0.05) for s in shapes]
            B.moe_pack_expert(f, hidden, inter, *(t.data_ptr() for t in w), None, None, None, blobs[e].data_ptr(), stream)
            dense.append([t.double() for t in w])
        else:
            q = [torch.randint(-127, 128, s, generator=g, device=DEV, dtype=torch.int32).to(I8) for s in shapes]
            sc = [((0.5 + torch.rand(s[0], generator=g, device=DEV)) * 7e-4).half() for s in shapes]
            B.moe_pack_expert(f, hidden, inter, *(t.data_ptr() for t in q), *(t.data_ptr() for t in sc), blobs[e].data_ptr(), stream)
            dense.append([a.double() * b.double()[:, None] for a, b in zip(q, sc)])
        torch.cuda.synchronize()
    return blobs, dense


def make_rows(g, fmt, n, hidden):
    if fmt == "bf16":
        x = normal(g, n, hidden, dtype=BF16)
        return x, None, x.double()
    q = torch.randint(-127, 128, (n, hidden), generator=g, device=DEV, dtype=torch.int32).to(I8)
    s = (0.5 + torch.rand(n, generator=g, device=DEV)) / 73
    return q, s, q.double() * s.double()[:, None]


def offsets_of(counts):
    return torch.tensor([0] + list(torch.tensor(counts).cumsum(0)), dtype=torch.int32, device=DEV)


COUNTS = [
    [1], [0, 1, 0], [16, 0, 17], [127, 129, 0, 1], [128, 256], [0, 0, 300, 5], [2] * 70, [33, 64, 31, 0, 257, 100, 1, 191]]


@pytest.mark.parametrize("counts", COUNTS)
@pytest.mark.parametrize("fmt,hidden,inter", [("bf16", 512, 64), ("bf16", 512, 1), ("bf16", 1024, 200), ("bf16", 2048, 129),
                                              ("int8", 1024, 8), ("int8", 1024, 136), ("int8", 2048, 64)])
def test_experts(lib, counts, fmt, hidden, inter):
    g = gen(sum(counts) + inter)
    n, tail = sum(counts), 3
    blobs, dense = make_blobs(lib, g, fmt, len(counts), hidden, inter)
    xs, scale, x = make_rows(g, fmt, n + tail, hidden)
    ys = lib.experts_rows(fmt, blobs, inter, xs, offsets_of(counts), scale=scale)
    assert not ys[n:].any()
    at = 0
    for c, (wg, wu, wd) in zip(counts, dense):
        r = x[at:at + c]
        a, b = r @ wg.t(), r @ wu.t()
        s = torch.sigmoid(a)
        h = a * s * b
        ref = h @ wd.t()
        # h: its own rounding and the sums behind it (their terms' sizes; d silu/da <= 1.1), 8-bit sums exact but for the scales
        sums = 64 * U32
        dh = U16 * h.abs() + sums * (1.1 * b.abs() * (r.abs() @ wg.abs().t()) + (a * s).abs() * (r.abs() @ wu.abs().t())) + 8 * U32 * h.abs()
        bound = 1.01 * (dh @ wd.abs().t()) + 64 * U32 * (h.abs() @ wd.abs().t()) + 1.01 * U16 * ref.abs()
        within(ys[at:at + c], ref, bound + 1e-12, "ys")
        at += c
    again = lib.experts_rows(fmt, blobs, inter, xs, offsets_of(counts), scale=scale)
    assert torch.equal(ys, again)


MANY = [300, 0, 1, 31, 257, 512, 96, 700, 33, 16] * 4  # (with these and a wide layer there are more tiles than compute units)


@pytest.mark.parametrize("fmt,hidden,inter", [("bf16", 1024, 1000), ("int8", 1024, 904), ("bf16", 2048, 897)])
def test_experts_many_tiles(lib, fmt, hidden, inter):
    g = gen(inter)
    blobs, dense = make_blobs(lib, g, fmt, len(MANY), hidden, inter)
    n = sum(MANY)
    xs, scale, x = make_rows(g, fmt, n + 5, hidden)
    ys = lib.experts_rows(fmt, blobs, inter, xs, offsets_of(MANY), scale=scale)
    assert not ys[n:].any()
    at = 0
    for e, (c, (wg, wu, wd)) in enumerate(zip(MANY, dense)):
        r = x[at:at + c]
        a, b = r @ wg.t(), r @ wu.t()
        s = torch.sigmoid(a)
        h = a * s * b
        ref = h @ wd.t()
        sums = 64 * U32
        dh = U16 * h.abs() + sums * (1.1 * b.abs() * (r.abs() @ wg.abs().t()) + (a * s).abs() * (r.abs() @ wu.abs().t())) + 8 * U32 * h.abs()
        within(ys[at:at + c], ref, 1.01 * (dh @ wd.abs().t()) + 64 * U32 * (h.abs() @ wd.abs().t()) + 1.01 * U16 * ref.abs() + 1e-12, f"ys {e}")
        at += c
    assert torch.equal(ys, lib.experts_rows(fmt, blobs, inter, xs, offsets_of(MANY), scale=scale))
    if fmt == "int8":
        return
    dys = normal(g, n + 5, hidden, dtype=BF16)
    again, kept = lib.experts_rows(fmt, blobs, inter, xs, offsets_of(MANY), keep=True)
    dxs, dblobs = lib.experts_rows_backward(fmt, blobs, inter, xs, offsets_of(MANY), kept, dys)
    assert torch.equal(again, ys) and not dxs[n:].any()
    dw = dblobs.view(BF16).view(len(MANY), inter, 3, hidden)
    at = 0
    for e, c in enumerate(MANY):
        if c == 0:
            assert not dw[e].any()
            continue
        leaves = [t.clone().requires_grad_() for t in (x[at:at + c], *dense[e])]
        grads = torch.autograd.grad(plain_expert(*leaves), leaves, dys[at:at + c].double())
        for got, ref, what in zip((dxs[at:at + c], dw[e, :, 0], dw[e, :, 1], dw[e, :, 2].t()), grads, ("dx", "dgate", "dup", "ddown")):
            off_ = float((got.double() - ref).norm() / ref.norm())
            assert off_ <= 6 * U16, (what, e, off_)
        at += c


def test_experts_more_tiles_than_a_list_holds(lib):
    """A workgroup lists 64 of its tiles at a time: gradients of many wide experts without rows but the last ones."""
    hidden, inter, experts = 4096, 64, 512
    g = gen(61)
    blobs = (torch.randn(experts, inter * 3 * hidden, generator=g, device=DEV) * 0.02).to(BF16).view(torch.uint8)
    counts = [0] * (experts - 3) + [5, 0, 70]
    xs, dys = normal(g, 75, hidden, dtype=BF16), normal(g, 75, hidden, dtype=BF16)
    ys, kept = lib.experts_rows("bf16", blobs, inter, xs, offsets_of(counts), keep=True)
    dxs, dblobs = lib.experts_rows_backward("bf16", blobs, inter, xs, offsets_of(counts), kept, dys)
    dw = dblobs.view(BF16).view(experts, inter, 3, hidden)
    assert not dw[:experts - 3].any() and not dw[experts - 2].any()
    for e, rows in ((experts - 3, slice(0, 5)), (experts - 1, slice(5, 75))):
        wg, wu, wd = blobs[e].view(BF16).view(inter, 3, hidden).double().unbind(1)
        leaves = [t.clone().requires_grad_() for t in (xs[rows].double(), wg, wu, wd.t())]
        y = plain_expert(*leaves)
        grads = torch.autograd.grad(y, leaves, dys[rows].double())
        for got, ref in ((ys[rows], y.detach()), (dxs[rows], grads[0]), (dw[e, :, 0], grads[1]), (dw[e, :, 1], grads[2]), (dw[e, :, 2].t(), grads[3])):
            assert float((got.double() - ref).norm() / ref.norm()) <= 6 * U16


def plain_expert(x, wg, wu, wd):
    a, b = x @ wg.t(), x @ wu.t()
    return (torch.nn.functional.silu(a) * b) @ wd.t()


@pytest.mark.parametrize("counts", COUNTS)
@pytest.mark.parametrize("hidden,inter", [(512, 64), (512, 1), (1024, 200), (2048, 129)])
def test_experts_backward(lib, counts, hidden, inter):
    g = gen(sum(counts) + inter + 1)
    n, tail = sum(counts), 2
    blobs, dense = make_blobs(lib, g, "bf16", len(counts), hidden, inter)
    xs, _, x = make_rows(g, "bf16", n + tail, hidden)
    dys = normal(g, n + tail, hidden, dtype=BF16)
    off = offsets_of(counts)
    ys, kept = lib.experts_rows("bf16", blobs, inter, xs, off, keep=True)
    assert torch.equal(ys, lib.experts_rows("bf16", blobs, inter, xs, off))
    dxs, dblobs = lib.experts_rows_backward("bf16", blobs, inter, xs, off, kept, dys)
    assert not dxs[n:].any()
    dw = dblobs.view(BF16).view(len(counts), inter, 3, hidden)
    at = 0
    for e, c in enumerate(counts):
        if c == 0:
            assert not dw[e].any()
            continue
        leaves = [t.clone().requires_grad_() for t in (x[at:at + c], *dense[e])]
        grads = torch.autograd.grad(plain_expert(*leaves), leaves, dys[at:at + c].double())
        mine = (dxs[at:at + c], dw[e, :, 0], dw[e, :, 1], dw[e, :, 2].t())
        for got, ref, what in zip(mine, grads, ("dx", "dgate", "dup", "ddown")):
            # g, u (through factors with slopes up to 1.1 and a curvature up to 0.5), their gradients and the result are rounded to
            # bf16: six roundings' worth over all elements
            off_ = float((got.double() - ref).norm() / ref.norm())
            assert off_ <= 6 * U16, (what, e, off_)
        at += c
    only, none = lib.experts_rows_backward("bf16", blobs, inter, xs, off, kept, dys, weights=False)
    assert none is None and torch.equal(only, dxs)
    none, only = lib.experts_rows_backward("bf16", blobs, inter, xs, off, kept, dys, rows=False)
    assert none is None and torch.equal(only, dblobs)


def test_experts_backward_against_differences(lib):
    g = gen(31)
    hidden, inter, c = 512, 96, 20
    blobs, dense = make_blobs(lib, g, "bf16", 1, hidden, inter)
    xs, _, x = make_rows(g, "bf16", c, hidden)
    dys = normal(g, c, hidden, dtype=BF16)
    _, kept = lib.experts_rows("bf16", blobs, inter, xs, offsets_of([c]), keep=True)
    dxs, dblobs = lib.experts_rows_backward("bf16", blobs, inter, xs, offsets_of([c]), kept, dys)
    dw = dblobs.view(BF16).view(inter, 3, hidden).double()
    args = [x, *dense[0]]
    grads = [dxs.double(), dw[:, 0], dw[:, 1], dw[:, 2].t()]
    for i in range(4):
        # along the gradient itself, so that nothing cancels
        v = grads[i] / grads[i].norm() * args[i].norm()
        e = 1e-5
        hi, lo = list(args), list(args)
        hi[i], lo[i] = args[i] + e * v, args[i] - e * v
        quotient = float(((plain_expert(*hi) - plain_expert(*lo)) * dys.double()).sum() / (2 * e))
        assert abs(quotient - float((grads[i] * v).sum())) <= 6 * U16 * abs(quotient), i


def test_experts_no_rows(lib):
    blobs, _ = make_blobs(lib, gen(1), "bf16", 2, 512, 16)
    off = torch.zeros(3, dtype=torch.int32, device=DEV)
    xs = torch.empty(0, 512, dtype=BF16, device=DEV)
    ys, kept = lib.experts_rows("bf16", blobs, 16, xs, off, keep=True)
    dxs, dblobs = lib.experts_rows_backward("bf16", blobs, 16, xs, off, kept, ys)
    assert ys.shape == (0, 512) and dxs.shape == (0, 512) and not dblobs.any()
    xs = normal(gen(2), 5, 512, dtype=BF16)  # (rows, but all of nobody)
    assert not lib.experts_rows("bf16", blobs, 16, xs, off).any()


def test_experts_keep_to_their_own_rows(lib):
    """What is not a number in one expert's rows or weights does not reach another's."""
    g = gen(41)
    counts = [40, 70, 30]
    blobs, _ = make_blobs(lib, g, "bf16", 3, 512, 40)
    xs, _, _ = make_rows(g, "bf16", 140, 512)
    dys = normal(g, 140, 512, dtype=BF16)
    off = offsets_of(counts)

    def both(b, x, d):
        ys, kept = lib.experts_rows("bf16", b, 40, x, off, keep=True)
        return ys, *lib.experts_rows_backward("bf16", b, 40, x, off, kept, d)

    ys, dxs, dw = both(blobs, xs, dys)
    bad_x, bad_b = xs.clone(), blobs.clone()
    bad_x[40:110] = float("nan")
    ys2, dxs2, dw2 = both(blobs, bad_x, dys)
    bad_b[1] = 0xff
    ys3, dxs3, dw3 = both(bad_b, xs, dys)
    for a, b in ((ys, ys2), (dxs, dxs2), (ys, ys3), (dxs, dxs3)):
        assert torch.equal(a[:40], b[:40]) and torch.equal(a[110:], b[110:]) and torch.isnan(b[40:110]).all()
    for b in (dw2, dw3):
        assert torch.equal(dw[0], b[0]) and torch.equal(dw[2], b[2])


# ---- together ---------------------------------------------------------------------------------------------------
def test_a_layer_in_a_graph_and_on_another_stream(lib):
    g = gen(51)
    T, K, E, d, I = 70, 4, 11, 1024, 72
    blobs, _ = make_blobs(lib, g, "int8", E, d, I)
    h, y = normal(g, T, d), normal(g, T, d, dtype=BF16)
    ids, weight = ids_of(g, T, K, E, 0.1), torch.rand(T, K, generator=g, device=DEV)

    def layer():
        n = lib.norm_rows(h, y, out=I8)
        o = lib.sort_tokens(ids, E)
        xs, scale = lib.gather_rows(n.x, o, scale=n.scale)
        return n.h, lib.combine_rows(lib.experts_rows("int8", blobs, I, xs, o.offsets, scale=scale), o, weight)

    ref = [t.clone() for t in layer()]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = layer()
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(ref, got))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = layer()
    for k in range(4):
        h.add_(0.25)
        ids.copy_(ids_of(g, T, K, E, 0.1 * k))
        ref = [t.clone() for t in layer()]
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(ref, out)), k
