"""Grids of launches over rows, on the CPU: every workgroup has its place, and HIP's limit of fewer than 2^32 threads along a
dimension holds for every number of rows that the operators take."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
X, MOST = 1 << 21, (1 << 26) - 1


def test_grids_hold_every_workgroup_within_the_limit(tmp_path):
    gxx = shutil.which("g++")
    if gxx is None:
        pytest.skip("no g++")
    exe = tmp_path / "row_grid"
    subprocess.run([gxx, "-std=c++17", "-O1", "-fsanitize=undefined", "-fno-sanitize-recover=all", "-static-libubsan", "-I",
                    os.path.join(ROOT, "paper_2412_00099_amd", "csrc"), os.path.join(ROOT, "tests", "host", "row_grid_driver.cpp"),
                    "-o", str(exe)], check=True, capture_output=True, text=True)
    groups = [1, 2, 1000, X - 1, X, X + 1, 3 * X, 3 * X + 7, 1 << 24, (1 << 24) + 1, 1 << 25, MOST // 4 + 1, MOST - 1, MOST]
    run = subprocess.run([str(exe)], input="\n".join(map(str, groups)), capture_output=True, text=True, check=True)
    lines = run.stdout.splitlines()
    assert len(lines) == len(groups)
    for n, line in zip(groups, lines):
        x, y = map(int, line.split())
        # (place of workgroup (i, j): j * X + i, so that a second line of them needs the first one whole)
        assert 1 <= x <= X and (y == 1 or x == X) and x * (y - 1) < n <= x * y, n
        assert x * 1024 < 1 << 32 and y < 1 << 16, n
