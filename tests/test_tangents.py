"""Forward-mode differentiation: the operators for tensors propagate no tangents, and say so where one would be lost.  The check comes
ahead of all others, so that tensors on the CPU will do."""
import pytest
import torch
import torch.autograd.forward_ad as fw

BF16, F32, I32 = torch.bfloat16, torch.float32, torch.int32
OFFSETS = torch.tensor([0, 4, 8], dtype=I32)


def calls():
    """(name, the operator, its floating-point inputs, called with them)"""
    import paper_2412_00099_amd as moe

    o = moe.TokenOrder(OFFSETS, torch.zeros(4, 2, dtype=I32), torch.zeros(8, dtype=I32))
    at, n = torch.tensor([0, 5], dtype=I32), torch.zeros(5, dtype=I32)
    rows = lambda h, t=BF16: torch.zeros(5, h, 64, dtype=t)  # noqa: E731
    pages, scale, table = torch.zeros(3, 2, 16, 64, dtype=torch.int8), torch.zeros(3, 2, 16), torch.zeros(5, 2, dtype=I32)
    wide, blobs = torch.zeros(3, 2, 16, 64, dtype=BF16), torch.zeros(2, 16, 3, 512, dtype=BF16)
    x8 = torch.zeros(8, 512, dtype=BF16)
    return [
        ("norm_rows", lambda h, y, gain: moe.norm_rows(h, y, gain), [torch.zeros(4, 8), torch.zeros(4, 8), torch.zeros(8)]),
        ("norm_rows_backward", moe.norm_rows_backward, [torch.zeros(4, 8), torch.zeros(8), torch.zeros(4), torch.zeros(4, 8), torch.zeros(4, 8)]),
        ("gather_rows", lambda x: moe.gather_rows(x, o), [torch.zeros(4, 8)]),
        ("combine_rows", lambda ys, w, base: moe.combine_rows(ys, o, w, base), [torch.zeros(8, 8), torch.zeros(4, 2), torch.zeros(4, 8)]),
        ("combine_rows_backward", lambda dy, ys, w: moe.combine_rows_backward(dy, ys, o, w), [torch.zeros(4, 8), torch.zeros(8, 8), torch.zeros(4, 2)]),
        ("experts_rows", lambda b, x: moe.experts_rows("bf16", b, 16, x, OFFSETS), [blobs, x8]),
        ("experts_rows_backward", lambda b, x, h, gu, dy: moe.experts_rows_backward("bf16", b, 16, x, OFFSETS, moe.KeptExperts(h, gu), dy),
         [blobs, x8, torch.zeros(8, 64, dtype=BF16), torch.zeros(8, 2, 64), x8]),
        ("store_pages", lambda k, v: moe.store_pages(k, v, n, wide, wide.clone()), [rows(2), rows(2)]),
        ("attend_pages", lambda q, k, v: moe.attend_pages(q, k, v, table, n), [rows(4), wide, wide]),
        ("attend_pages, 8 bits", lambda q, ks, vs: moe.attend_pages(q, pages, pages, table, n, ks, vs), [rows(4), scale, scale]),
        ("attend_rows", lambda q, k, v: moe.attend_rows(q, k, v, at), [rows(4), rows(2), rows(2)]),
        ("attend_rows_backward", lambda q, k, v, y, lse, low, dy: moe.attend_rows_backward(q, k, v, at, y, moe.KeptAttention(lse, low), dy),
         [rows(4), rows(2), rows(2), rows(4), torch.zeros(4, 5), rows(4), rows(4)]),
    ]


def test_tangents_are_not_lost_in_silence():
    for name, call, inputs in calls():
        for i in range(len(inputs)):
            with fw.dual_level():
                dual = [fw.make_dual(x, torch.ones_like(x)) if i == j else x for j, x in enumerate(inputs)]
                with pytest.raises(ValueError, match="tangent"):
                    call(*dual)
                with torch.no_grad(), pytest.raises(ValueError, match="tangent"):
                    call(*dual)
                with pytest.raises(ValueError, match="GPU"):  # (as far as the next check)
                    call(*[fw.unpack_dual(x).primal for x in dual])


def test_a_function_with_a_jvp_of_its_own_may_call_them():
    """Its forward runs without tangents."""
    for name, call, inputs in calls():
        class Own(torch.autograd.Function):
            @staticmethod
            def forward(*xs):
                with pytest.raises(ValueError, match="GPU"):
                    call(*xs)
                return xs[0] * 2

            @staticmethod
            def setup_context(ctx, inputs, output):
                pass

            @staticmethod
            def jvp(ctx, *tangents):
                return tangents[0] * 2

        with fw.dual_level():
            y = Own.apply(*[fw.make_dual(x, torch.ones_like(x)) for x in inputs])
            assert bool((fw.unpack_dual(y).tangent == 2).all()), name


def test_a_tangent_of_a_level_that_is_over_is_none():
    for name, call, inputs in calls():
        with fw.dual_level():
            duals = [fw.make_dual(x, torch.ones_like(x)) for x in inputs]
        with pytest.raises(ValueError, match="GPU"):
            call(*duals)
