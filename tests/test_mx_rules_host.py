"""The rules by which the microscaled and layer norm calls shape their launches, looked at without a GPU."""
from __future__ import annotations

import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2510_11400_amd", "csrc")


def _program(folder, body, header):
    cxx = shutil.which("g++") or shutil.which("c++")
    if not cxx:
        pytest.skip("no C++ compiler")
    src, exe = str(folder / "rules.cpp"), str(folder / "rules")
    with open(src, "w") as f:
        f.write(f'#include "{header}"\n#include <cstdio>\nint main()\n{{\n    long long a, b, c;\n    {body}\n}}\n')
    subprocess.run([cxx, "-std=c++17", "-I", CSRC, src, "-o", exe], check=True)
    return lambda rows: [tuple(int(v) for v in line.split()) for line in subprocess.run(
        [exe], input="".join(" ".join(map(str, r)) + "\n" for r in rows), text=True, check=True, capture_output=True).stdout.splitlines()]


def test_a_launch_has_fewer_threads_than_its_limit(tmp_path):
    """The dimensions' product stays under 2^32, also where one workgroup of 256 threads a chunk of 256 columns takes a whole row of 2^31 of them."""
    at_once = _program(tmp_path, 'while (std::scanf("%lld", &a) == 1) std::printf("%lld\\n", (long long)fh::groups_at_once(a));', "fh_rules.hpp")
    threads = [64, 256, 512, 1000, 1024, 3 * 256, 12345 * 256, 2 ** 23 * 256, 2 ** 23 * 256 + 1]
    for t, (n,) in zip(threads, at_once([(t,) for t in threads])):
        assert n >= 1 and (n * t <= 2 ** 31 and (n + 1) * t > 2 ** 31 or n == 1)
        # a third dimension, from 65535 groups on, makes it up to 65534 groups more
        assert (n + (65534 if n > 65535 else 0)) * t < 2 ** 32
    # parts of whole groups of 32 rows where a workgroup of 1024 takes one
    assert at_once([(1024,)]) == [(2 ** 21,)]
