"""The gated projection without a GPU: what the workspaces' sizes refuse, and gelu's polynomial as it stands in the source."""
from __future__ import annotations

import os
import re

import numpy as np
import pytest
import torch
from scipy.special import erfcx

from paper_2510_11400_amd import api

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.parametrize("size", [api.gated_workspace_bytes, api.gated_backward_workspace_bytes])
def test_sizes_of_workspaces_are_of_operands_in_device_memory(size):
    x = torch.zeros(4, 40)
    with pytest.raises(ValueError, match="device memory"):
        size(x, x, x)
    with pytest.raises(TypeError, match="must be a tensor"):
        size(x.numpy(), x, x)


def test_gelus_tail_is_fitted_relative_to_its_size():
    """R(x) = Phi(-x) e^(x^2/2) by the polynomial in 1/(1 + p x), evaluated in 64 bits from the constants' binary32 values, up to where the power in front of it leaves binary32
    (e^(-x^2/2) < 2^-126 from 13.22 on), and finite behind.  Bound: the fit 2.7e-7; coefficients off by 2^-24 each, their terms' magnitudes at most twice the value, 1.2e-7; p off by
    2^-24, of which t takes x p / (1 + x p) and R 1.4 times that where the former is near 1, 0.8e-7."""
    with open(os.path.join(ROOT, "paper_2510_11400_amd", "csrc", "fh_activation.hpp")) as f:
        source = f.read()
    tail = np.array([np.float32(v) for v in re.search(r"kTail\[8\] = \{([^}]*)\}", source).group(1).replace("f", "").split(",")], dtype=np.float64)
    p = float(np.float32(re.search(r"__builtin_fabsf\(g\), ([0-9.]+)f, 1\.0f", source).group(1)))
    assert tail.size == 8

    def fitted(x):
        t = 1.0 / (1.0 + p * x)
        return np.polynomial.polynomial.polyval(t, tail)

    x = np.concatenate((np.linspace(0.0, 13.22, 200001), np.logspace(-8, 1, 1001)))
    assert np.max(np.abs(fitted(x) / (0.5 * erfcx(x / np.sqrt(2.0))) - 1.0)) <= 4.7e-7
    assert np.all(np.abs(fitted(np.logspace(1.1, 38, 1001))) < 0.04)
