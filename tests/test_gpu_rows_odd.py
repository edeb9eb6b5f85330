"""Row operators at widths and addresses that leave a part of a unit of 8 columns at a row's end, also where a result takes the
place of an input: against the same operators in 64 bits, and in place against not in place, bit for bit."""
import pytest
import torch

from test_gpu_rows import BF16, DEV, F32, I8, U16, U32, gen, ids_of, normal, within

pytestmark = pytest.mark.gpu
WIDTHS = [3, 8, 9, 15, 63, 65, 519, 1031, 2047, 4099, 8191]


def at_offset(t, elements):
    """A copy of t whose first element lies `elements` behind an aligned address."""
    space = torch.empty(t.numel() + elements, dtype=t.dtype, device=t.device)
    out = space[elements:].view(t.shape)
    out.copy_(t)
    return out


@pytest.mark.parametrize("d", WIDTHS)
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_norm_in_place_and_off_the_grid(lib, d, dtype):
    from paper_2412_00099_amd import binding as B
    g = gen(d)
    fmt = {F32: B.MOE_R_FP32, BF16: B.MOE_R_BF16}[dtype]
    h, y, gain = normal(g, 33, d, dtype=dtype), normal(g, 33, d, dtype=BF16), 1 + normal(g, d, std=0.2)
    ref = {out: lib.norm_rows(h, y, gain, out=out) for out in (F32, BF16, I8)}
    s = ref[F32].h.double()
    rstd = (s.square().mean(1, keepdim=True) + 1e-6).rsqrt()
    within(ref[F32].x, s * rstd * gain.double(), (s * rstd * gain.double()).abs() * 64 * U32, "x")
    for off in (1, 5):
        for out in (F32, BF16, I8):
            n = lib.norm_rows(at_offset(h, off), at_offset(y, off), at_offset(gain, off), out=out)
            assert torch.equal(n.h, ref[out].h) and torch.equal(n.x, ref[out].x)
            mine, x = at_offset(h, off), at_offset(torch.zeros(33, d, device=DEV, dtype=out), off)
            scale = torch.empty(33, device=DEV)
            B.moe_norm_rows(mine.data_ptr(), fmt, d, y.data_ptr(), B.MOE_R_BF16, d, gain.data_ptr(), 1e-6, 33, d, mine.data_ptr(), x.data_ptr(),
                            {F32: B.MOE_R_FP32, BF16: B.MOE_R_BF16, I8: B.MOE_R_INT8}[out], scale.data_ptr() if out == I8 else None, None,
                            torch.cuda.current_stream().cuda_stream)
            assert torch.equal(mine, ref[out].h) and torch.equal(x, ref[out].x)


@pytest.mark.parametrize("d", WIDTHS)
def test_norm_backward_in_place(lib, d):
    from paper_2412_00099_amd import binding as B
    g = gen(d + 1)
    h, gain, dx, dh = normal(g, 700, d), 1 + normal(g, d, std=0.2), normal(g, 700, d, dtype=BF16), normal(g, 700, d)
    n = lib.norm_rows(h, None, gain)
    got, dgain = lib.norm_rows_backward(h, gain, n.rstd, dx, dh)
    leaf, gl = h.double().requires_grad_(), gain.double().requires_grad_()
    x = leaf * (leaf.square().mean(1, keepdim=True) + 1e-6).rsqrt() * gl
    want, wgain = torch.autograd.grad((x * dx.double()).sum() + (leaf * dh.double()).sum(), [leaf, gl])
    size = n.rstd.double()[:, None] * ((dx.double() * gain.double()).abs() + (h.double() * n.rstd.double()[:, None]).abs()
                                       * (dx.double() * gain.double() * h.double() * n.rstd.double()[:, None]).abs().mean(1, keepdim=True)) + dh.double().abs()
    within(got, want, 128 * U32 * size, "dh")
    within(dgain, wgain, 128 * U32 * (dx.double() * h.double() * n.rstd.double()[:, None]).abs().sum(0), "dgain")
    mine, dg = at_offset(dh, 3), torch.empty_like(gain)
    need = B.moe_norm_rows_backward_bytes(700, d)
    work = torch.empty(need, dtype=torch.uint8, device=DEV)
    B.moe_norm_rows_backward(h.data_ptr(), B.MOE_R_FP32, gain.data_ptr(), n.rstd.data_ptr(), dx.data_ptr(), B.MOE_R_BF16, mine.data_ptr(), 700, d,
                             mine.data_ptr(), dg.data_ptr(), work.data_ptr(), need, torch.cuda.current_stream().cuda_stream)
    assert torch.equal(mine, got) and torch.equal(dg, dgain)


@pytest.mark.parametrize("d", WIDTHS)
@pytest.mark.parametrize("ys_type,y_type", [(BF16, F32), (F32, BF16)])
def test_order_in_place_and_off_the_grid(lib, d, ys_type, y_type):
    from paper_2412_00099_amd import binding as B
    g = gen(d + 2)
    ids = ids_of(g, 50, 3, 7, 0.2)
    o = lib.sort_tokens(ids, 7)
    used = int(o.offsets[-1])
    ys, w, base = normal(g, 150, d, dtype=ys_type), torch.rand(50, 3, generator=g, device=DEV), normal(g, 50, d, dtype=y_type)
    ys[used:] = float("nan")  # rows of nobody
    ref = lib.combine_rows(ys, o, w, base)
    row = o.row_of.long()
    rows = torch.where((row >= 0)[..., None], ys.double()[row.clamp(min=0)], 0.0) * w.double()[..., None]
    want = base.double() + rows.sum(1)
    within(ref, want, 64 * U32 * (base.double().abs() + rows.abs().sum(1)) + (0 if y_type == F32 else 1.01 * U16) * want.abs(), "y")
    mine = at_offset(base, 1)
    fmts = {F32: B.MOE_R_FP32, BF16: B.MOE_R_BF16}
    off = at_offset(ys, 3)
    B.moe_combine_rows(off.data_ptr(), fmts[ys_type], o.row_of.data_ptr(), w.data_ptr(), mine.data_ptr(), 50, 3, d, mine.data_ptr(), fmts[y_type],
                       torch.cuda.current_stream().cuda_stream)
    assert torch.equal(mine, ref)

    dy = normal(g, 50, d, dtype=y_type)
    dys, dw = lib.combine_rows_backward(dy, ys, o, w)
    terms = torch.where((row >= 0)[..., None], ys.double()[row.clamp(min=0)], 0.0) * dy.double()[:, None]
    within(dw, terms.sum(2), 64 * U32 * terms.abs().sum(2), "dweight")
    again, dw2 = lib.combine_rows_backward(at_offset(dy, 1), off, o, w)
    assert torch.equal(dys, again) and torch.equal(dw, dw2) and not dys[used:].any()

    for x in (dy, dy.to(torch.int8)):
        xs, _ = lib.gather_rows(x, o)
        odd, _ = lib.gather_rows(at_offset(x, 1), o)
        token = o.entry_of[:used].long() // 3
        assert torch.equal(xs[:used], x[token]) and not xs[used:].any() and torch.equal(xs, odd)
