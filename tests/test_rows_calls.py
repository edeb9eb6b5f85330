"""How the operators on many rows are called, as far as that shows without a GPU: what their tensors' part refuses."""
import pytest
import torch


@pytest.fixture(scope="module")
def moe():
    import paper_2412_00099_amd

    return paper_2412_00099_amd


OFFSETS = torch.zeros(3, dtype=torch.int32)


@pytest.mark.parametrize("fmt,blob", [("bf16", torch.float32), ("bf16", torch.float16), ("int8", torch.bfloat16), ("int8", torch.int32)])
def test_blobs_are_bytes_or_the_weights_type(moe, fmt, blob):
    """Large enough in bytes is not enough: numbers of another type are no packed experts."""
    xs = torch.zeros(4, 1024, dtype=torch.int8 if fmt == "int8" else torch.bfloat16)
    blobs = torch.zeros(2, 16, 3, 1024, dtype=blob)
    with pytest.raises(ValueError, match="blobs"):
        moe.experts_rows(fmt, blobs, 16, xs, OFFSETS)


def needing(*shape, dtype=torch.float32):
    return torch.zeros(*shape, dtype=dtype, requires_grad=True)


@pytest.mark.parametrize("call", [
    lambda moe, o: moe.norm_rows(needing(4, 8)),
    lambda moe, o: moe.norm_rows(torch.zeros(4, 8), needing(4, 8)),
    lambda moe, o: moe.norm_rows(torch.zeros(4, 8), None, needing(8)),
    lambda moe, o: moe.norm_rows_backward(torch.zeros(4, 8), torch.zeros(8), torch.zeros(4), needing(4, 8)),
    lambda moe, o: moe.gather_rows(needing(4, 8), o),
    lambda moe, o: moe.combine_rows(needing(8, 8), o),
    lambda moe, o: moe.combine_rows(torch.zeros(8, 8), o, needing(4, 2)),
    lambda moe, o: moe.combine_rows(torch.zeros(8, 8), o, None, needing(4, 8)),
    lambda moe, o: moe.combine_rows_backward(needing(4, 8), torch.zeros(8, 8), o),
    lambda moe, o: moe.experts_rows("bf16", needing(2, 16, 3, 512, dtype=torch.bfloat16), 16, torch.zeros(8, 512, dtype=torch.bfloat16), o.offsets),
    lambda moe, o: moe.experts_rows("bf16", torch.zeros(2, 16, 3, 512, dtype=torch.bfloat16), 16, needing(8, 512, dtype=torch.bfloat16), o.offsets),
])
def test_gradients_are_not_lost_in_silence(moe, call):
    """The calls record nothing for automatic differentiation: where that would lose a gradient they say so."""
    o = moe.TokenOrder(OFFSETS, torch.zeros(4, 2, dtype=torch.int32), torch.zeros(8, dtype=torch.int32))
    with pytest.raises(ValueError, match="gradient"):
        call(moe, o)
    with torch.no_grad(), pytest.raises(ValueError, match="GPU"):  # (as far as the next check)
        call(moe, o)
