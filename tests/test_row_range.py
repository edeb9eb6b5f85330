"""The rows between two offsets, on the CPU: whatever the offsets hold, the rows are among those that there are, and their number does
not pass 32 bits on the way."""
import itertools
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LEAST, MOST = -(1 << 31), (1 << 31) - 1


def test_rows_between_offsets_are_rows_that_there_are(tmp_path):
    gxx = shutil.which("g++")
    if gxx is None:
        pytest.skip("no g++")
    exe = tmp_path / "row_range"
    subprocess.run([gxx, "-std=c++17", "-O1", "-fsanitize=undefined", "-fno-sanitize-recover=all", "-static-libubsan", "-I",
                    os.path.join(ROOT, "paper_2412_00099_amd", "csrc"), os.path.join(ROOT, "tests", "host", "row_range_driver.cpp"),
                    "-o", str(exe)], check=True, capture_output=True, text=True)
    ends = [LEAST, LEAST + 1, LEAST + 150, -200, -1, 0, 1, 20, 150, 199, 200, 201, (1 << 26) - 1, 1 << 30, MOST - 1, MOST]
    cases = list(itertools.product(ends, ends, (0, 1, 200, (1 << 26) - 1)))
    run = subprocess.run([str(exe)], input="\n".join("%d %d %d" % c for c in cases), capture_output=True, text=True, check=True)
    lines = run.stdout.splitlines()
    assert len(lines) == len(cases)
    for (a, b, rows), line in zip(cases, lines):
        first, count = map(int, line.split())
        assert first == min(max(a, 0), rows), (a, b, rows)
        assert count == max(min(max(b, 0), rows) - first, 0), (a, b, rows)
        assert 0 <= first <= first + count <= rows, (a, b, rows)


def test_a_difference_of_the_ends_as_they_are_would_wrap():
    """What an end that is cut to the rows from above alone makes of (150, the least number): 2^31 - 150 rows."""
    end = min(LEAST, 200)
    assert (end - 150 + (1 << 31)) % (1 << 32) - (1 << 31) == 2147483498
