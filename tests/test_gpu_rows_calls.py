"""How the operators on many rows are called, at sizes and layouts that the numerical tests do not have."""
import pytest
import torch

from test_gpu_rows import BF16, DEV, F32, gen, make_blobs, normal, offsets_of

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("what", ["experts", "most experts", "top_k", "hidden", "inter"])
def test_sizes_are_refused_before_memory_is_taken(lib, what):
    ids = torch.zeros(4096, 2, dtype=torch.int32, device=DEV)
    order = lib.sort_tokens(ids, 2)
    wide = lib.TokenOrder(order.offsets, torch.zeros(4096, 64, dtype=torch.int32, device=DEV), order.entry_of)
    x = torch.zeros(4096, 1024, dtype=BF16, device=DEV)
    blobs = torch.zeros(2, lib.moe_blob_bytes(lib.MOE_W_BF16, 1024, 16), dtype=torch.uint8, device=DEV)
    call = {"experts": lambda: lib.sort_tokens(ids, 1 << 20),
            "most experts": lambda: lib.sort_tokens(ids, (1 << 31) - 1),
            "top_k": lambda: lib.gather_rows(x, wide),
            "hidden": lambda: lib.norm_rows(x.view(256, 16384)),
            "inter": lambda: lib.experts_rows("bf16", blobs, 1 << 16, x, order.offsets, keep=True)}[what]
    torch.cuda.synchronize()
    torch.cuda.reset_peak_memory_stats()
    before = torch.cuda.memory_allocated()
    with pytest.raises(lib.MoEError):
        call()
    assert torch.cuda.max_memory_allocated() - before < 1 << 16


@pytest.mark.parametrize("dtype", [torch.uint8, BF16])
def test_what_lies_between_blobs_has_no_gradient(lib, dtype):
    """Blobs may lie further apart than they are long; what the caching allocator hands out for the gradients is not zero."""
    g = gen(1)
    hidden, inter, counts = 1024, 200, [5, 0, 40]
    packed, _ = make_blobs(lib, g, "bf16", 3, hidden, inter)
    n = packed.shape[1]
    blobs = torch.full((3, n + 512), 7, dtype=torch.uint8, device=DEV)
    blobs[:, :n] = packed
    xs, dys = normal(g, 45, hidden, dtype=BF16), normal(g, 45, hidden, dtype=BF16)
    ys, kept = lib.experts_rows("bf16", blobs, inter, xs, offsets_of(counts), keep=True)
    _, want = lib.experts_rows_backward("bf16", packed, inter, xs, offsets_of(counts), kept, dys, rows=False)
    full = [torch.full_like(blobs, 0xff) for _ in range(3)]
    torch.cuda.synchronize()
    del full
    _, got = lib.experts_rows_backward("bf16", blobs.view(dtype), inter, xs, offsets_of(counts), kept, dys, rows=False)
    assert got.dtype == dtype
    got = got.view(torch.uint8)
    assert torch.equal(got[:, :n], want) and not got[:, n:].any()


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_gradient_of_rows_that_lie_apart(lib, dtype):
    """norm_rows takes rows with a stride, and without y hands them back: its backward takes what it returns."""
    g = gen(2)
    h, gain, dx = normal(g, 70, 900, dtype=dtype)[:, 3:703], 1 + normal(g, 700, std=0.2), normal(g, 70, 700, dtype=BF16)
    n = lib.norm_rows(h, gain=gain)
    assert torch.equal(n.h, h)
    got, want = (lib.norm_rows_backward(t, gain, n.rstd, dx) for t in (n.h, h.contiguous()))
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    with pytest.raises(ValueError):
        lib.norm_rows_backward(h.t().contiguous().t(), gain, n.rstd, dx)
