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
