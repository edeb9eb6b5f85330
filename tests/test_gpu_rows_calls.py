"""How the operators on many rows are called, at sizes and layouts that the numerical tests do not have."""
import pytest
import torch

from test_gpu_rows import BF16, DEV

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
