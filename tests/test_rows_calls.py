"""How the operators on many rows are called, as far as that shows without a GPU: what their tensors' part refuses, and what works
where it has not been built."""
import importlib.util
import os
import subprocess
import sys

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


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


WITHOUT = """
import sys

class Missing:
    def find_spec(self, name, path=None, target=None):
        if name == "paper_2412_00099_amd._rows":
            raise ImportError("no such library")

sys.meta_path.insert(0, Missing())
import paper_2412_00099_amd as moe
assert moe.moe_blob_bytes(moe.MOE_W_BF16, 512, 8) and moe.MoEDecoder and moe.ExpertStore
for name in ("norm_rows", "experts_rows", "TokenOrder"):
    try:
        getattr(moe, name)
    except ImportError as e:
        assert "build.py" in str(e)
    else:
        raise SystemExit(name)
try:
    moe.something_else
except AttributeError:
    print("fine")
"""


def test_decode_needs_no_tensors_part():
    run = subprocess.run([sys.executable, "-c", WITHOUT], cwd=ROOT, capture_output=True, text=True, timeout=120)
    assert run.returncode == 0 and run.stdout.split() == ["fine"], run.stderr[-2000:]


def test_the_library_is_built_without_a_host_compiler(tmp_path, monkeypatch):
    spec = importlib.util.spec_from_file_location("build_of_a_test", os.path.join(ROOT, "paper_2412_00099_amd", "build.py"))
    build = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(build)
    if not os.path.exists(os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")):
        pytest.skip("no hipcc")
    monkeypatch.setattr(build, "SOURCES", {"trace_sim.hip": []})
    monkeypatch.setattr(build, "OUT", str(tmp_path / "libmoe_cache.so"))
    monkeypatch.setattr(build, "TENSORS_OUT", str(tmp_path / "_rows.so"))
    monkeypatch.setattr(build, "OBJ_DIR", str(tmp_path))
    monkeypatch.setenv("CXX", str(tmp_path / "no-such-compiler"))
    with pytest.raises(RuntimeError, match="row operators"):
        build.build(verbose=False)
    assert os.path.exists(tmp_path / "libmoe_cache.so") and not os.path.exists(tmp_path / "_rows.so")
