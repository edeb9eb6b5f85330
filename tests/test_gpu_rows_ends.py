"""Experts whose rows end far below zero: the difference of such offsets passes 32 bits (its arithmetic: test_row_range.py)."""
import pytest
import torch

from test_gpu_rows import DEV, gen, make_blobs, make_rows, normal

pytestmark = pytest.mark.gpu
LEAST = -(1 << 31)


@pytest.mark.parametrize("n,hidden,inter", [(60, 512, 64), (700, 1024, 200), (3000, 512, 129)])
def test_an_end_far_below_zero_is_of_no_rows(lib, n, hidden, inter):
    """The other experts' products and weights' gradients are what they are without it."""
    g = gen(n)
    blobs, _ = make_blobs(lib, g, "bf16", 2, hidden, inter)
    xs, _, _ = make_rows(g, "bf16", n + 5, hidden)
    dys = normal(g, n + 5, hidden, dtype=torch.bfloat16)
    out = []
    for end in (n, LEAST, LEAST + 7):
        offsets = torch.tensor([0, n, end], dtype=torch.int32, device=DEV)
        _, kept = lib.experts_rows("bf16", blobs, inter, xs, offsets, keep=True)
        _, dblobs = lib.experts_rows_backward("bf16", blobs, inter, xs, offsets, kept, dys)
        torch.cuda.synchronize()
        out.append((kept.h[:n], dblobs))
    for h, dblobs in out[1:]:
        assert torch.equal(h, out[0][0]) and torch.equal(dblobs, out[0][1])
