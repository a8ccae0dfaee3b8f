"""Inline assembly in the kernels' sources: what it writes without the compiler's knowledge is named as clobbered."""
from __future__ import annotations

import glob
import os
import re

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _statements():
    for path in sorted(glob.glob(os.path.join(ROOT, "paper_2510_11400_amd", "csrc", "*.h*"))):
        with open(path) as f:
            text = f.read()
        for m in re.finditer(r"\basm(?:\s+volatile)?\s*\((.*?)\);", text, re.S):
            yield os.path.basename(path), m.group(1)


def test_registers_that_assembly_moves_into_are_clobbered():
    """m0 and the like: the compiler may hold a value of its own there."""
    seen = 0
    for path, text in _statements():
        code, *parts = re.split(r"\n?\s*:(?!:)|::", text)
        for register in re.findall(r"\bs_mov_b32 (m0|vcc_lo|vcc_hi|exec_lo|exec_hi)", code):
            seen += 1
            assert f'"{register}"' in parts[-1], f"{path}: {text}"
    assert seen > 0
