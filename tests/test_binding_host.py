"""The package without its compiled binding, in a copy of its own: what ctypes reaches still works, the rest says what is missing."""
from __future__ import annotations

import os
import shutil
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

PROGRAM = """
import sys
sys.path.insert(0, sys.argv[1])
import torch
from paper_2510_11400_amd import api, hooks, layers, workloads
assert api.__file__.startswith(sys.argv[1]), api.__file__
assert api.packed_bytes(1024, 4) == api.raw_library().fh_packed_bytes(1024, 4) > 0 and api.raw_library().fh_mx_bytes(4, 40) == api.mx_bytes(4, 40)
hooks.SavedActivations(256, 4)
x = torch.zeros(4, 40)
for call in (lambda: api.fh_mx_quantize(x), lambda: api.fh_layer_norm(x), lambda: layers.mx_linear(x, x), lambda: layers.layer_norm(x),
             lambda: api.MxLayer(x, x).forward()):
    try:
        call()
    except ImportError as e:
        assert "_fh_binding" in str(e) and "build" in str(e), e
    else:
        raise AssertionError("no error")
print("fine")
"""


@pytest.mark.parametrize("binding", ["missing", "of something else"])
def test_the_older_calls_do_without_the_binding(tmp_path, binding):
    shutil.copytree(os.path.join(ROOT, "paper_2510_11400_amd"), tmp_path / "paper_2510_11400_amd",
                    ignore=shutil.ignore_patterns("_build", "csrc", "_fh_binding.so", "__pycache__"))
    if binding != "missing":
        (tmp_path / "paper_2510_11400_amd" / "_fh_binding.so").write_bytes(b"no library")
    done = subprocess.run([sys.executable, "-c", PROGRAM, str(tmp_path)], capture_output=True, text=True, cwd=tmp_path)
    assert done.returncode == 0 and done.stdout == "fine\n", done.stderr
