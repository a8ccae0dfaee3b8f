"""The rules by which the microscaled and layer norm calls shape their launches, looked at without a GPU."""
from __future__ import annotations

import ctypes
import os
import shutil
import subprocess

import pytest

import mx_products as M
from paper_2510_11400_amd import api

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


def _plans(tmp_path):
    """plans(rows of m, n, k) -> (kernel, parts of the sum, chunks a part, whether tiles of 64 go in runs)"""
    return _program(tmp_path, '''while (std::scanf("%lld %lld %lld", &a, &b, &c) == 3) {
        const fh::Plan p = fh::plan_of(a, b, (c + 255) / 256);
        std::printf("%d %d %lld %d\\n", (int)p.tile, (int)p.parts, (long long)p.chunks_each, (int)fh::tiles_in_runs(a, b, (c + 255) / 256));
    }''', "fh_mx_plan.hpp")


def test_the_tested_products_take_the_kernels_that_they_test(tmp_path):
    got = _plans(tmp_path)([shape for _, _, *shape in M.PRODUCTS])
    for (kernel, how, *shape), (tile, parts, _, runs) in zip(M.PRODUCTS, got):
        assert M.KERNELS[tile] == kernel, shape
        assert (parts > 1) == (how == M.SPLIT), shape
        if kernel == "waves64":
            assert bool(runs) == (how == M.RUNS), shape
    assert {(kernel, how) for kernel, how, *_ in M.PRODUCTS} == {("waves32", None), ("waves32_wide", None), ("waves32_wide", M.SPLIT), ("waves64", M.RUNS),
                                                                  ("waves64", M.ORDER), ("square128", None), ("square256", None)}


def test_a_sums_parts_make_up_the_sum(tmp_path):
    """Every chunk is in one part, none is empty, and the workspace that the library asks for holds a product for each."""
    shapes = [(m, n, k) for m in (1, 31, 96, 130, 1000) for n in (1, 64, 97) for k in (0, 1, 256, 8191, 8192, 8200, 40000, 1 << 20, 1 << 24)]
    split = 0
    for (m, n, k), (_, parts, each, _) in zip(shapes, _plans(tmp_path)(shapes)):
        chunks = (k + 255) // 256
        assert parts >= 1 and parts * each >= chunks and (parts - 1) * each < max(chunks, 1)
        assert api.mx_matmul_workspace_bytes(m, n, k) == (parts * m * n * 4 if parts > 1 else 0)
        split += parts > 1
    assert split > 20


def test_a_split_product_is_refused_without_its_workspace():
    m, n, k = 96, 97, 40000
    need = api.mx_matmul_workspace_bytes(m, n, k)
    fake, big = 0x10000, 1 << 40                                          # never dereferenced: the call is refused first
    assert need > 0
    for pointer, cap, status in ((None, big, 1), (fake, need - 1, 7), (fake + 4, big, 8)):
        p = api.fh_mx_product(fake, big, fake, big, m, n, k, None, 0, 0, fake, n, big, pointer, cap, 0)
        assert api.raw_library().fh_mx_matmul(ctypes.byref(p), None) == status
