"""Compile the HIP sources into paper_2412_00099_amd/libmoe_cache.so (gfx950 only, in-tree), and the tensors' part of the row
operators (host code only) into _rows.so beside it."""
from __future__ import annotations

import os
import subprocess
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(HERE, "csrc")
OUT = os.path.join(HERE, "libmoe_cache.so")
TENSORS_OUT = os.path.join(HERE, "_rows.so")
OBJ_DIR = os.path.join(HERE, "_build")

COMMON = [
    "--offload-arch=gfx950",
    "-O3",
    "-fPIC",
    "-std=c++17",
    "-I" + os.path.join(ROOT, "include"),
    "-I" + CSRC,
    "-Wall",
    "-Wno-unused-function",
    # packed fp32 VALU forms are not to be generated on the test machines
    "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
    "-fhip-fp32-correctly-rounded-divide-sqrt",
    # the first 16 words of a kernel's scalar arguments arrive in registers: no load at its start (0.3 us a launch)
    "-mllvm", "-amdgpu-kernarg-preload-count=16",
]
# per-file extras: the routing decisions are single-rounding fp32 steps, so no contraction there
SOURCES = {
    "router.hip": ["-ffp-contract=off"],
    "expert_gemv.hip": [],
    "expert_gemv_quant.hip": [],
    "pack.hip": [],
    "moe_cache.hip": [],
    "trace_sim.hip": [],
    "expert_static.hip": [],
    "expert_batch.hip": [],
    "rows_norm.hip": ["-ffp-contract=off"],  # (8-bit codes are decided by single-rounding steps)
    "rows_order.hip": [],
    "rows_experts.hip": [],
    "rows_api.hip": [],
}


def _torch() -> str:
    import importlib.util

    spec = importlib.util.find_spec("torch")
    if spec is None:
        raise RuntimeError("PyTorch is not installed")
    return os.path.dirname(spec.origin)


def _tensors_command(obj: str) -> list[str]:
    """csrc/rows_torch.cpp to an object file"""
    import sysconfig

    return [os.environ.get("CXX", "g++"), "-c", os.path.join(CSRC, "rows_torch.cpp"), "-o", obj, "-O2", "-std=c++17", "-fPIC", "-fvisibility=hidden",
            "-Wall", "-DUSE_ROCM=1", "-D__HIP_PLATFORM_AMD__=1", "-I" + os.path.join(ROOT, "include"), "-isystem", os.path.join(_torch(), "include"),
            "-isystem", "/opt/rocm/include", "-I" + sysconfig.get_paths()["include"]]


def _tensors_link(obj: str) -> list[str]:
    libs = os.path.join(_torch(), "lib")
    return [os.environ.get("CXX", "g++"), "-shared", "-o", TENSORS_OUT, obj, "-L" + os.path.dirname(OUT), "-l:libmoe_cache.so", "-L" + libs,
            "-ltorch_python", "-ltorch", "-ltorch_cpu", "-lc10", "-lc10_hip", "-Wl,-rpath,$ORIGIN", "-Wl,-rpath," + libs]


def _start(cmd: list[str], verbose: bool) -> subprocess.Popen:
    if verbose:
        print("[build]", " ".join(cmd), flush=True)
    return subprocess.Popen(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)


def _done(what: str, p: subprocess.Popen, verbose: bool) -> bool:
    out, _ = p.communicate()
    out = "\n".join(l for l in out.splitlines() if "packed-fp32-ops" not in l and l.strip())
    if out and verbose:
        print(out)
    if p.returncode != 0:
        print(f"[build] {what} failed", file=sys.stderr)
    return p.returncode == 0


def build(verbose: bool = True) -> str:
    """The library, and then the tensors' part of the row operators, which also needs a host compiler and PyTorch's headers: without
    them the library is there all the same, and the error says what is not."""
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    os.makedirs(OBJ_DIR, exist_ok=True)
    objs = [os.path.join(OBJ_DIR, src + ".o") for src in SOURCES]
    procs = [(src, _start([hipcc, "-c", os.path.join(CSRC, src), "-o", obj] + COMMON + extra, verbose))
             for (src, extra), obj in zip(SOURCES.items(), objs)]
    tensors_obj, tensors, missing = os.path.join(OBJ_DIR, "rows_torch.cpp.o"), None, "a compiler failed"
    try:
        tensors = _start(_tensors_command(tensors_obj), verbose)
    except (OSError, RuntimeError) as e:
        missing = str(e)
    compiled = [_done(src, p, verbose) for src, p in procs]
    tensors_compiled = tensors is not None and _done("rows_torch.cpp", tensors, verbose)
    if not all(compiled):
        raise RuntimeError("hipcc failed")
    cmd = [hipcc, "-shared", "-fPIC", "--offload-arch=gfx950", "-o", OUT] + objs
    if verbose:
        print("[build]", " ".join(cmd), flush=True)
    subprocess.check_call(cmd)
    if not tensors_compiled or not _done("_rows.so", _start(_tensors_link(tensors_obj), verbose), verbose):
        raise RuntimeError(f"{OUT} is built, the row operators for tensors are not: {missing}")
    return OUT


if __name__ == "__main__":
    build()
