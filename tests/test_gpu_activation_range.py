"""The gated projection's activations where their factor s is small, relative to their own size, and at the ends of the range.

One feature, an input of 1 and weights that are the gates: the kernel's gate is the weight itself, and up is 1 by its bias.

Bounds, in half steps of fp32 (2^-24 of the value).  A power of a rounded argument a is off by r |a| for r roundings on the way to a (constants count), and by 2 for the
instruction; a reciprocal by 2.
  silu        a = g, r = 2; the power, an addition, the reciprocal and the product with g are 6 at most
  gelu_tanh   a = 2 z, r = 8 (the cubic term's constant, two products, the sum, two more constants with their products); the same 6
  gelu        a = g^2/2, r = 3; beside the power s has a polynomial P(t), t = 1/(1 + p |g|).  t is off by 4 (its constant, the sum, the reciprocal), which R(g) = Phi(-g) e^(g^2/2)
              takes 2.3 times at most (at g = 0, where R'/R is 0.8 and p 0.348); seven steps of a polynomial whose terms' magnitudes add up to twice its value at most
              are 14, its coefficients 2, its fit 4.5; the power's instruction, its product and that with g 4
"""
from __future__ import annotations

import math

import pytest

torch = pytest.importorskip("torch")
import gated_reference as R  # noqa: E402

pytestmark = pytest.mark.gpu

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
STEP = 2.0 ** -24


@pytest.fixture(scope="module")
def api():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a visible MI355X")
    from paper_2510_11400_amd import api as _api
    return _api


def _factors(g, act):
    """(half steps of the power behind s, of s beside it)"""
    if act == "silu":
        return 2 * g.abs(), 6.0
    if act == "gelu":
        return 1.5 * g * g, 34.0
    return 8 * math.sqrt(8.0 / math.pi) * (g + 0.044715 * g ** 3).abs(), 6.0


def _one_feature(g, tokens, dtype):
    """(x, w_gate, w_up, b_gate, b_up): every token's gates are g, its ups 1."""
    n = g.numel()
    return (torch.ones(tokens, 1, device="cuda", dtype=dtype), g.to(dtype).view(n, 1).cuda(), torch.zeros(n, 1, device="cuda", dtype=dtype),
            None, torch.ones(n, device="cuda", dtype=dtype))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("tokens", [1, 40, 300])
@pytest.mark.parametrize("act, least", [("silu", -80.0), ("gelu", -12.5), ("gelu_tanh", -9.0)])
def test_the_lower_tail_relative_to_its_size(api, act, least, tokens, dtype):
    parts = _one_feature(torch.linspace(least, 0.0, 2001), tokens, DTYPES[dtype])
    g = parts[1].double().view(1, -1)
    want = R.activation(g, act)[0].expand(tokens, -1)
    power, beside = _factors(g, act)
    bound = want.abs() * ((power + beside) * STEP + (R.HALF[DTYPES[dtype]] if dtype == "bf16" else 0.0))
    R.check(api.fh_gated(*parts, act), want, bound, act)


@pytest.mark.parametrize("act, least", [("silu", -80.0), ("gelu", -12.5), ("gelu_tanh", -9.0)])
def test_the_slopes_lower_tail(api, act, least):
    """The bias's gradient for one token whose result's gradient is 1: s + g s'.  s is off as above; s' = s (1 - s) z' takes that once more by 1 - s, at most as much
    where s is up to 1/2, and eight roundings."""
    parts = _one_feature(torch.linspace(least, 0.0, 2001), 1, torch.float32)
    g = parts[1].double().view(-1)
    dh = torch.ones(1, g.numel(), device="cuda")
    got = api.fh_gated_backward(dh, *parts[:3], torch.zeros_like(parts[4]), parts[4], act, needs_input=False)[3]
    want = R.activation(g, act)[1]
    s = R.activation(g, act)[0] / g.clamp(max=-1e-30)
    s[-1] = 0.5
    power, beside = _factors(g, act)
    bound = STEP * ((power + beside) * s + (2 * (power + beside) + 8.0) * (want - s).abs() + want.abs())
    R.check(got, want, bound, act)


@pytest.mark.parametrize("act", ["silu", "gelu", "gelu_tanh"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_gates_up_to_the_end_of_the_range(api, act, dtype):
    """From 1e6 to 3.4e38 either way: the activation is g or 0, its slope 1 or 0, whatever its powers do on the way."""
    size = torch.logspace(6, 38.5, 651)
    parts = _one_feature(torch.cat((size, -size)), 1, DTYPES[dtype])
    g = parts[1].double().view(1, -1)
    want = torch.where(g > 0, g, 0.0)
    assert torch.equal(api.fh_gated(*parts, act).double(), want)
    dh = torch.ones(1, g.numel(), device="cuda", dtype=DTYPES[dtype])
    _, dw_gate, dw_up, db_gate, db_up = api.fh_gated_backward(dh, *parts[:3], torch.zeros_like(parts[4]), parts[4], act, needs_input=False)
    assert torch.equal(db_gate.double(), (g[0] > 0).double()) and torch.equal(dw_gate[:, 0], db_gate)
    assert torch.equal(db_up.double(), want[0]) and torch.equal(dw_up[:, 0], db_up)
