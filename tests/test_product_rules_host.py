"""The rules by which a product of rows in chunks of 128 bytes takes its kernel, looked at without a GPU."""
from __future__ import annotations

import os
import shutil
import subprocess

import pytest

import q8_gated_shapes as S

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2510_11400_amd", "csrc")


def _program(folder, body):
    cxx = shutil.which("g++") or shutil.which("c++")
    if not cxx:
        pytest.skip("no C++ compiler")
    src, exe = str(folder / "rules.cpp"), str(folder / "rules")
    with open(src, "w") as f:
        f.write(f'#include "fh_product_plan.hpp"\n#include <cstdio>\nint main()\n{{\n    long long a, b, c, d, e, f;\n    {body}\n}}\n')
    subprocess.run([cxx, "-std=c++17", "-I", CSRC, src, "-o", exe], check=True)
    return lambda rows: [tuple(int(v) for v in line.split()) for line in subprocess.run(
        [exe], input="".join(" ".join(map(str, r)) + "\n" for r in rows), text=True, check=True, capture_output=True).stdout.splitlines()]


@pytest.fixture(scope="module")
def plans(tmp_path_factory):
    """plans(rows of m, n, chunks, fp32, shared, with rests) -> (kernel, parts, chunks a part, side, rows of a sum of columns)"""
    run = _program(tmp_path_factory.mktemp("rules"), '''while (std::scanf("%lld %lld %lld %lld %lld %lld", &a, &b, &c, &d, &e, &f) == 6) {
        const fh::ProductPlan p = fh::product_plan(a, b, c, d != 0, e != 0, fh::product_last(f != 0));
        std::printf("%d %u %u %lld %lld\\n", (int)p.tile, p.parts, p.chunks_each, (long long)fh::product_side(p.tile), (long long)fh::product_sum_rows(p.tile));
    }''')
    return lambda rows: run([(*r, 0) if len(r) == 5 else r for r in rows])


@pytest.fixture(scope="module")
def few(tmp_path_factory):
    return _program(tmp_path_factory.mktemp("few"), '''while (std::scanf("%lld %lld", &a, &b) == 2)
        std::printf("%d %d %d\\n", (int)fh::few_rows_of_bytes(a, b != 0), (int)fh::few_rows_dense(a, true, false), (int)fh::few_rows_dense(a, false, b != 0));''')


def test_the_tested_shapes_take_every_kernel(plans, few):
    for shapes, times, pair in ((S.PRODUCTS, 1, 0), (S.GATED, 2, 1)):
        taken = [f[0] for f in few([(m, pair) for m, _, _ in shapes])]
        tiles = {p[0] for p, f in zip(plans([(m, times * n, -(-k // 128), 0, 0) for m, n, k in shapes]), taken) if not f}
        assert sorted(tiles) == list(range(5)) and any(taken), (pair, tiles)
    for dtype in ("bf16", "f32"):
        rows = [(dtype, *s[:3]) for s in S.DENSE + S.STRIDED] + [s for s in S.LARGE if s[0] == dtype]
        of = {name: {(p[0], p[1] > 1) for p in plans([S.products_of(*r)[name] for r in rows])} for name in ("pair", "dx", "dw")}
        assert {t for t, _ in of["pair"]} == set(range(5)) and {t for t, _ in of["dx"]} == set(range(5)), (dtype, of)
        shared = {t for t, parts in of["dw"] if parts}
        assert shared == (set(range(5)) if dtype == "bf16" else {0, 1, 2}), (dtype, of)
        assert {t for t, _ in of["dw"]} >= {0, 1, 2, 3}, (dtype, of)


def test_a_sums_parts_make_up_the_sum(plans):
    """Every chunk is in one part, none is empty; only sums that may be shared are."""
    shapes = [(m, n, c, slow, shared) for m in (1, 33, 130, 1000, 5000) for n in (1, 64, 97, 3000) for c in (1, 2, 8, 17, 128, 1000, 32768) for slow in (0, 1) for shared in (0, 1)]
    for (m, n, c, _, shared), (_, parts, each, _, _) in zip(shapes, plans(shapes)):
        assert parts >= 1 and parts * each >= c and (parts - 1) * each < c
        assert parts == 1 or shared
    assert plans([(5, 7, 0, 0, 0)])[0][:3] == (0, 1, 0)


def test_sums_of_columns_stand_for_the_rows_of_a_workgroup_or_of_half_a_tile(plans):
    got = {p[0]: p[3:] for p in plans([(m, n, c, s, 0) for m in (1, 100, 3000, 9000) for n in (16, 900, 6000) for c in (1, 8, 40) for s in (0, 1)])}
    assert got == {0: (32, 32), 1: (32, 32), 2: (64, 64), 3: (128, 64), 4: (256, 128)}


def test_few_rows(few):
    """In 8 bits up to 4 rows and up to 8 of a pair, fp32 up to 16, bf16 where its operands would have to be laid out."""
    rows = [(m, pair) for m in (1, 4, 5, 8, 9, 16, 17) for pair in (0, 1)]
    for (m, flag), (of_bytes, fp32, bf16) in zip(rows, few(rows)):
        assert of_bytes == (m <= (8 if flag else 4)) and fp32 == (m <= 16) and bf16 == (m <= 16 and flag)


def test_rests_are_kept_of_few_gradients_in_bf16(tmp_path, plans):
    run = _program(tmp_path, 'while (std::scanf("%lld %lld %lld %lld", &a, &b, &c, &d) == 4) std::printf("%d\\n", (int)fh::product_with_rests(a, b, c, d != 0));')
    rows = [(1, 1, 1, 0), (1, 1, 1, 1), (512, 256, 1024, 0), (512, 257, 1024, 0), (512, 1, 1025, 0), (512, 256, 512, 1), (1 << 21, 1, 1, 0), (1 << 19, 256, 1, 0),
            (1 << 21, 1 << 20, 1 << 20, 0)]
    assert [r[0] for r in run(rows)] == [1, 0, 1, 0, 0, 0, 0, 1, 0]
    shapes = [S.products_of("bf16", *s) for s in S.WITH_RESTS]
    assert all(p["dx"][5] for p in shapes)
    taken = {name: {p[0] for p in plans([s[name] for s in shapes])} for name in ("pair", "dx", "dw")}
    assert taken["pair"] == {0, 1} and taken["dx"] == {0, 1, 2} and taken["dw"] == {0, 1, 2}, taken
    assert {p[1] > 1 for p in plans([s["dw"] for s in shapes])} == {False, True}
