"""What the operators on many rows refuse: every check comes before the GPU is touched, so the pointers here are never read."""
import ctypes as C

import pytest
import torch


@pytest.fixture(scope="module")
def B():
    from paper_2412_00099_amd import binding

    return binding


P = 0x10000  # never dereferenced


def refused(B, call, good, **bad):
    args = dict(good, **bad)
    code = call(*args.values())
    assert code == B.MOE_EINVAL, (bad, code)
    assert B.moe_last_error()


NORM = dict(h=P, h_fmt=0, h_stride=64, y=P, y_fmt=1, y_stride=64, gain=P, eps=1e-6, n_rows=3, hidden=64, h_out=2 * P, x=P, x_fmt=1, scale=None,
            rstd=None, stream=None)


@pytest.mark.parametrize("bad", [
    dict(h=None), dict(x=None), dict(h_fmt=2), dict(y_fmt=2), dict(x_fmt=3), dict(h_fmt=-1), dict(hidden=0), dict(hidden=8193), dict(n_rows=-1),
    dict(n_rows=1 << 26), dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf")), dict(h_stride=63), dict(y_stride=10), dict(h_out=None),
    dict(h_out=P, h_stride=65), dict(x_fmt=2), dict(scale=P), dict(h=P + 2), dict(y=P + 1), dict(gain=P + 2), dict(rstd=P + 1)])
def test_norm(B, bad):
    refused(B, B.lib.moe_norm_rows, NORM, **bad)


BACK = dict(h=P, h_fmt=0, gain=P, rstd=P, dx=P, x_fmt=1, dh_in=None, n_rows=3, hidden=64, dh=P, dgain=P, work=P, work_bytes=1 << 20, stream=None)


@pytest.mark.parametrize("bad", [dict(h=None), dict(rstd=None), dict(dx=None), dict(dh=None), dict(x_fmt=2), dict(h_fmt=2), dict(hidden=0),
                                 dict(n_rows=-5), dict(work=None), dict(work_bytes=64 * 4 * 3 - 1), dict(work=P + 4), dict(dh_in=P + 1)])
def test_norm_backward(B, bad):
    refused(B, B.lib.moe_norm_rows_backward, BACK, **bad)


SORT = dict(ids=P, n_tokens=40000, top_k=4, n_experts=60, offsets=P, row_of=P, entry_of=P, work=P, work_bytes=1 << 20, stream=None)


@pytest.mark.parametrize("bad", [dict(ids=None), dict(offsets=None), dict(row_of=None), dict(entry_of=None), dict(top_k=0), dict(top_k=9),
                                 dict(n_experts=0), dict(n_experts=513), dict(n_tokens=-1), dict(n_tokens=1 << 25), dict(work=None),
                                 dict(work_bytes=8), dict(ids=P + 2)])
def test_sort(B, bad):
    refused(B, B.lib.moe_sort_tokens, SORT, **bad)


GATHER = dict(x=P, fmt=1, x_stride=64, scale=None, row_of=P, offsets=P, n_tokens=4, top_k=2, n_experts=8, hidden=64, xs=P, xs_scale=None,
              stream=None)


@pytest.mark.parametrize("bad", [dict(x=None), dict(xs=None), dict(row_of=None), dict(offsets=None), dict(fmt=3), dict(x_stride=63),
                                 dict(scale=P), dict(xs_scale=P), dict(hidden=0), dict(x=P + 1), dict(top_k=9)])
def test_gather(B, bad):
    refused(B, B.lib.moe_gather_rows, GATHER, **bad)


COMBINE = dict(ys=P, ys_fmt=1, row_of=P, weight=None, base=None, n_tokens=4, top_k=2, hidden=64, y=P, y_fmt=0, stream=None)


@pytest.mark.parametrize("bad", [dict(ys=None), dict(y=None), dict(row_of=None), dict(ys_fmt=2), dict(y_fmt=2), dict(hidden=9000), dict(top_k=0),
                                 dict(weight=P + 2), dict(base=P + 2)])
def test_combine(B, bad):
    refused(B, B.lib.moe_combine_rows, COMBINE, **bad)


CBACK = dict(dy=P, dy_fmt=0, ys=P, ys_fmt=1, row_of=P, offsets=P, weight=None, n_tokens=4, top_k=2, n_experts=8, hidden=64, dys=P, dweight=P,
             stream=None)


@pytest.mark.parametrize("bad", [dict(dy=None), dict(ys=None), dict(dys=None), dict(offsets=None), dict(dy_fmt=2), dict(ys_fmt=2),
                                 dict(n_experts=0), dict(n_tokens=-1)])
def test_combine_backward(B, bad):
    refused(B, B.lib.moe_combine_rows_backward, CBACK, **bad)


EXPERTS = dict(fmt=1, hidden=512, inter=64, n_experts=4, blobs=P, stride=512 * 64 * 6, xs=P, scale=None, offsets=P, n_rows=9, h=P, gu=None, ys=P,
               stream=None)


@pytest.mark.parametrize("bad", [dict(fmt=0), dict(fmt=3), dict(fmt=9), dict(hidden=100), dict(inter=0), dict(n_experts=0), dict(n_experts=513),
                                 dict(blobs=None), dict(stride=512 * 64 * 6 - 16), dict(stride=512 * 64 * 6 + 8), dict(xs=None), dict(scale=P),
                                 dict(offsets=None), dict(n_rows=-1), dict(h=None), dict(ys=None), dict(xs=P + 8), dict(blobs=P + 4),
                                 dict(hidden=4096, inter=1 << 20, stride=1 << 40)])
def test_experts(B, bad):
    refused(B, B.lib.moe_experts_rows, EXPERTS, **bad)


def test_experts_int8_needs_scales(B):
    refused(B, B.lib.moe_experts_rows, EXPERTS, fmt=2, hidden=1024, stride=1 << 20)


EBACK = dict(fmt=1, hidden=512, inter=64, n_experts=4, blobs=P, stride=512 * 64 * 6, xs=P, offsets=P, n_rows=9, h=P, gu=P, dys=P, dgu=P, dxs=P,
             dblobs=P, stream=None)


@pytest.mark.parametrize("bad", [dict(fmt=2), dict(fmt=0), dict(gu=None), dict(h=None), dict(dys=None), dict(dgu=None), dict(xs=None),
                                 dict(dxs=P + 8), dict(hidden=500)])
def test_experts_backward(B, bad):
    refused(B, B.lib.moe_experts_rows_backward, EBACK, **bad)


def test_workspace_sizes(B):
    assert B.moe_sort_tokens_bytes(0, 4, 60) == 0 and B.moe_sort_tokens_bytes(8, 4, 60) == 0
    assert B.moe_sort_tokens_bytes(40000, 4, 60) > 0
    assert B.moe_norm_rows_backward_bytes(0, 64) == 0 and B.moe_norm_rows_backward_bytes(3, 64) == 3 * 64 * 4
    assert B.moe_norm_rows_backward_bytes(3, 8193) == 0


def test_tensors_have_to_be_on_a_gpu_and_fit():
    import paper_2412_00099_amd as moe

    with pytest.raises(ValueError):
        moe.norm_rows(torch.zeros(2, 8))
    with pytest.raises(ValueError):
        moe.norm_rows(torch.zeros(2, 8), torch.zeros(3, 8))
    with pytest.raises(ValueError):
        moe.norm_rows(torch.zeros(8, 2).t())
    with pytest.raises(ValueError):
        moe.norm_rows(torch.zeros(2, 8, dtype=torch.float64))
    with pytest.raises(ValueError):
        moe.sort_tokens(torch.zeros(4, 2, dtype=torch.int64), 8)
    o = moe.TokenOrder(torch.zeros(9, dtype=torch.int32), torch.zeros(4, 2, dtype=torch.int32), torch.zeros(8, dtype=torch.int32))
    for call in (lambda: moe.gather_rows(torch.zeros(5, 8), o), lambda: moe.combine_rows(torch.zeros(7, 8), o),
                 lambda: moe.combine_rows(torch.zeros(8, 8), o, weight=torch.zeros(4, 3)),
                 lambda: moe.combine_rows_backward(torch.zeros(4, 8), torch.zeros(8, 9), o),
                 lambda: moe.experts_rows("bf16", torch.zeros(7, 10, dtype=torch.uint8), 4, torch.zeros(8, 512, dtype=torch.bfloat16), o.offsets),
                 lambda: moe.experts_rows("bf16", torch.zeros(8, 10, dtype=torch.uint8), 4, torch.zeros(8, 512), o.offsets)):
        with pytest.raises(ValueError):
            call()
