"""The gated projection of dense matrices, its backward pass and its layers on the GPU, within the roundings' bounds (gated_reference)."""
from __future__ import annotations

import pytest

torch = pytest.importorskip("torch")
import gated_reference as R  # noqa: E402
import q8_gated_shapes as S  # noqa: E402

pytestmark = pytest.mark.gpu

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
ACTIVATIONS = ("silu", "gelu", "gelu_tanh")


@pytest.fixture(scope="module")
def api():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a visible MI355X")
    from paper_2510_11400_amd import api as _api
    return _api


@pytest.fixture(scope="module")
def layers(api):
    from paper_2510_11400_amd import layers as _layers
    return _layers


def _inputs(t, k, f, dtype, bias=True, seed=0):
    """(x, w_gate, w_up, b_gate, b_up, dh); rows of several sizes, gates from far below zero to far above."""
    g = torch.Generator().manual_seed(seed + t + 3 * k + 7 * f)

    def normal(*shape):
        return torch.randn(shape, generator=g)

    x = normal(t, k) * torch.exp2(torch.randint(-2, 3, (t, 1), generator=g).float())
    parts = [x, normal(f, k) / k ** 0.5, normal(f, k) / k ** 0.5, normal(f) if bias else None, normal(f) if bias else None,
             normal(t, f) * 1e-3 * torch.exp(normal(t, 1))]
    return [None if p is None else p.to(dtype).cuda() for p in parts]


def _check_gated(api, x, wg, wu, bg, bu, act, out=None):
    h, bound = R.gated(R.dense_product(x, wg, bg), R.dense_product(x, wu, bu), act, x.dtype)
    got = api.fh_gated(x, wg, wu, bg, bu, act, out=out)
    R.check(got, h, bound, (tuple(x.shape), tuple(wg.shape), act))
    return got


def _check_backward(api, dh, x, wg, wu, bg, bu, act, **kind):
    want = R.gated_backward(dh, x, wg, wu, bg, bu, act)
    got = api.fh_gated_backward(dh, x, wg, wu, bg, bu, act, **kind)
    for name, y, (w, bound) in zip(("dx", "dw_gate", "dw_up", "db_gate", "db_up"), got, want):
        if y is not None:
            assert y.dtype == x.dtype
            R.check(y, w, bound, (name, tuple(x.shape), tuple(wg.shape), act))
    return got


@pytest.mark.parametrize("act", ACTIVATIONS)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("t, k, f", S.DENSE)
def test_gated(api, t, k, f, dtype, act):
    x, wg, wu, bg, bu, _ = _inputs(t, k, f, DTYPES[dtype])
    got = _check_gated(api, x, wg, wu, bg, bu, act)
    assert torch.equal(got, api.fh_gated(x, wg, wu, bg, bu, act))
    _check_gated(api, x, wg, wu, None, bu, act)


@pytest.mark.parametrize("act", ACTIVATIONS)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("t, k, f", S.DENSE)
def test_backward(api, t, k, f, dtype, act):
    x, wg, wu, bg, bu, dh = _inputs(t, k, f, DTYPES[dtype])
    got = _check_backward(api, dh, x, wg, wu, bg, bu, act)
    again = api.fh_gated_backward(dh, x, wg, wu, bg, bu, act)
    assert all(torch.equal(a, b) for a, b in zip(got, again))


@pytest.mark.parametrize("act", ACTIVATIONS)
@pytest.mark.parametrize("t, k, f", S.WITH_RESTS)
def test_small_backward_passes_keep_the_rests_of_a_rounding(api, t, k, f, act):
    """Up to 2^19 gradients of the gates and 2^27 products of theirs: the products take each with its rounding's rest.  A bf16 value is off by 2^-8 of it at most, its rest by 2^-8 of that:
    2^-16 in all, and the sums have twice as many terms."""
    x, wg, wu, bg, bu, dh = _inputs(t, k, f, torch.bfloat16)
    want = R.gated_backward(dh, x, wg, wu, bg, bu, act, rests=True)
    got = api.fh_gated_backward(dh, x, wg, wu, bg, bu, act)
    for name, y, (w, bound) in zip(("dx", "dw_gate", "dw_up", "db_gate", "db_up"), got, want):
        R.check(y, w, bound, (name, t, k, f, act))


def test_rests_of_what_is_no_number(api):
    """Gradients beyond bf16's range and NaN: the results that they reach are no numbers, the others are as without them."""
    x, wg, wu, bg, bu, dh = _inputs(40, 64, 50, torch.bfloat16)
    want = api.fh_gated_backward(dh, x, wg, wu, bg, bu, "silu")
    dh[3, 7], dh[20, 0] = float("nan"), float("inf")
    got = api.fh_gated_backward(dh, x, wg, wu, bg, bu, "silu")
    rest = [i for i in range(40) if i not in (3, 20)]
    assert not bool(torch.isfinite(got[0][[3, 20]]).any()) and torch.equal(got[0][rest], want[0][rest])
    cols = [i for i in range(50) if i not in (0, 7)]
    for g, w in zip(got[1:], want[1:]):
        assert not bool(torch.isfinite(g[[0, 7]]).any()) and torch.equal(g[cols], w[cols])


@pytest.mark.parametrize("dtype, t, k, f", S.LARGE)
def test_large(api, dtype, t, k, f):
    x, wg, wu, bg, bu, dh = _inputs(t, k, f, DTYPES[dtype])
    _check_gated(api, x, wg, wu, bg, bu, "gelu")
    got = _check_backward(api, dh, x, wg, wu, bg, bu, "gelu")
    again = api.fh_gated_backward(dh, x, wg, wu, bg, bu, "gelu")
    assert all(torch.equal(a, b) for a, b in zip(got, again))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("t, k, f", [(70, 48, 30), (300, 100, 128), (3000, 64, 300)])
def test_gradients_wherever_the_caller_wants_them(api, dtype, t, k, f):
    """By the C call the weights' gradients lie apart, in either order, or one behind the other: the same values, and nothing else is written."""
    import ctypes
    x, wg, wu, bg, bu, dh = _inputs(t, k, f, DTYPES[dtype])
    want = api.fh_gated_backward(dh, x, wg, wu, bg, bu, "silu")
    n = f * k
    for first, second in ((16, 16 + n), (16, 16 + n + 8), (16 + n + 24, 16)):
        room = torch.full((2 * n + 64,), 7.0, device="cuda", dtype=x.dtype)
        l = api.fh_gated_layer(t, k, f, int(dtype == "bf16"), 0, api.FH_GATED_NEEDS_WEIGHT, 0, x.data_ptr(), k, wg.data_ptr(), k, wu.data_ptr(), k, bg.data_ptr(), bu.data_ptr(),
                               None, f, 0, dh.data_ptr(), f)
        l.dw_gate, l.dw_up = (room.data_ptr() + at * room.element_size() for at in (first, second))
        need = api.raw_library().fh_gated_workspace_bytes(ctypes.byref(l), 1)
        workspace = torch.full((need + 64,), 170, dtype=torch.uint8, device="cuda")
        l.workspace, l.workspace_cap = workspace.data_ptr(), need
        assert api.raw_library().fh_gated_backward(ctypes.byref(l), ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)) == 0
        assert torch.equal(room[first:first + n].view(f, k), want[1]) and torch.equal(room[second:second + n].view(f, k), want[2])
        room[first:first + n] = 7.0
        room[second:second + n] = 7.0
        assert bool((room == 7.0).all()) and bool((workspace[need:] == 170).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_backward_of_what_is_asked_for(api, dtype):
    """Every subset gives the same gradients; those of biases that are not there are None."""
    x, wg, wu, bg, bu, dh = _inputs(130, 72, 100, DTYPES[dtype])
    whole = _check_backward(api, dh, x, wg, wu, bg, bu, "silu")
    for input in (False, True):
        for weight in (False, True):
            for bias in (False, True):
                some = api.fh_gated_backward(dh, x, wg, wu, bg, bu, "silu", needs_input=input, needs_weight=weight, needs_bias=bias)
                for y, w, wanted in zip(some, whole, (input, weight, weight, bias, bias)):
                    assert (y is not None) == wanted and (y is None or torch.equal(y, w))
    one = _check_backward(api, dh, x, wg, wu, bg, None, "silu")
    assert one[3] is not None and one[4] is None
    none = _check_backward(api, dh, x, wg, wu, None, None, "silu")
    assert none[3] is None and none[4] is None


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows", [3, 40, 300])
def test_strided_and_unaligned_operands(api, dtype, rows):
    """Views of larger matrices at every alignment: what lies around them is neither read into the results nor written."""
    x, wg, wu, bg, bu, dh = _inputs(rows, 200, 150, DTYPES[dtype])

    def view(t, rows, cols, at, extra):
        whole = torch.full((rows, cols + extra), float("nan"), device="cuda", dtype=t.dtype)
        whole[:, at:at + cols] = t[:rows, :cols]
        return whole[:, at:at + cols]

    for k, f, at, extra in ((200, 150, 0, 56), (192, 128, 8, 64), (128, 96, 1, 3), (64, 150, 3, 8), (199, 149, 5, 11), (128, 64, 2, 126)):
        parts = [view(x, rows, k, at, extra), view(wg, f, k, at, extra), view(wu, f, k, (at + 4) % (extra + 1), extra)]
        biases = [view(b[None], 1, f, at, extra)[0] for b in (bg, bu)]
        out = torch.full((rows, f + 7), 7.0, device="cuda", dtype=x.dtype)
        _check_gated(api, *parts, *biases, "silu", out=out[:, 3:3 + f])
        assert bool((out[:, :3] == 7.0).all()) and bool((out[:, 3 + f:] == 7.0).all())
        _check_backward(api, view(dh, rows, f, at, extra), *parts, *biases, "gelu")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("t, k, f, extra", S.STRIDED)
def test_strided_operands_of_large_products(api, t, k, f, dtype, extra):
    """Rows at multiples of 16 bytes that are none of 128, whole chunks and parts of them."""
    x, wg, wu, bg, bu, dh = _inputs(t, k, f, DTYPES[dtype])

    def view(m, extra):
        whole = torch.full((m.shape[0], m.shape[1] + extra), float("nan"), device="cuda", dtype=m.dtype)
        whole[:, :m.shape[1]] = m
        return whole[:, :m.shape[1]]

    parts = [view(x, extra), view(wg, 2 * extra), view(wu, 0)]
    _check_gated(api, *parts, bg, bu, "silu")
    _check_backward(api, view(dh, 3), *parts, bg, bu, "silu")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_rows_without_numbers(api, dtype):
    """A NaN in a token reaches its own results, and the weights' gradients, which are sums over all tokens."""
    x, wg, wu, bg, bu, dh = _inputs(70, 96, 40, DTYPES[dtype])
    clean = api.fh_gated(x, wg, wu, bg, bu)
    clean_dx = api.fh_gated_backward(dh, x, wg, wu, bg, bu)[0]
    x[5, 3] = float("nan")
    h = api.fh_gated(x, wg, wu, bg, bu)
    others = torch.arange(70, device="cuda") != 5
    assert bool(torch.isnan(h[5]).all()) and torch.equal(h[others], clean[others])
    dx, dwg, dwu, dbg, dbu = api.fh_gated_backward(dh, x, wg, wu, bg, bu)
    assert bool(torch.isnan(dx[5]).all()) and torch.equal(dx[others], clean_dx[others])
    assert all(bool(torch.isnan(d).all()) for d in (dwg, dwu, dbg, dbu))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_no_tokens(api, dtype):
    x, wg, wu, bg, bu, dh = _inputs(0, 33, 20, DTYPES[dtype])
    assert api.fh_gated(x, wg, wu, bg, bu).shape == (0, 20)
    dx, *sums = api.fh_gated_backward(dh, x, wg, wu, bg, bu)
    assert dx.shape == (0, 33) and all(not bool(s.any()) and s.numel() for s in sums)


@pytest.mark.parametrize("act", ACTIVATIONS)
def test_activations_over_their_range(api, act):
    """The gate alone, from -1e18 (whose cube is out of range) to 1e18 and around zero: one feature, unit weights, up is 1."""
    g = torch.cat((torch.linspace(-12, 12, 4001), torch.logspace(-30, 18, 700), -torch.logspace(-30, 18, 700), torch.tensor([0.0, -0.0])))
    n = g.numel()
    x = torch.ones(1, 1, device="cuda")
    wg, bu = g.view(n, 1).cuda(), torch.ones(n, device="cuda")
    wu = torch.zeros(n, 1, device="cuda")
    _check_gated(api, x, wg, wu, None, bu, act)
    dh = torch.ones(1, n, device="cuda")
    _check_backward(api, dh, x, wg, wu, None, bu, act)


@pytest.mark.parametrize("act", ACTIVATIONS)
def test_gradients_against_differences(api, act):
    """Along random directions the gradients' products agree with differences of the definition in 64 bits.  The difference is off by a third
    derivative's h^2, the gradients by their bounds' sums; both are far below the 1e-3 of the largest that is asked for."""
    parts = _inputs(40, 50, 30, torch.float32)
    inputs, dh = parts[:5], parts[5]
    grads = api.fh_gated_backward(dh, *inputs, act)

    def loss(values):
        x, wg, wu, bg, bu = values
        return float((dh.double() * R.activation(R.mm(x, wg.t()) + bg, act)[0] * (R.mm(x, wu.t()) + bu)).sum())

    g = torch.Generator(device="cuda").manual_seed(5)
    for i, grad in enumerate(grads):
        for _ in range(3):
            v = torch.randn(grad.shape, generator=g, device="cuda", dtype=torch.float64)
            at = [p.double() for p in inputs]
            step = 1e-5
            values = []
            for sign in (1, -1):
                moved = list(at)
                moved[i] = at[i] + sign * step * v
                values.append(loss(moved))
            slope = (values[0] - values[1]) / (2 * step)
            assert abs(slope - float((grad.double() * v).sum())) <= 1e-3 * float(grad.double().norm() * v.norm()) / v.numel() ** 0.5


def test_refusals(api):
    x, wg, wu, bg, bu, dh = _inputs(6, 20, 10, torch.float32)
    with pytest.raises(ValueError, match="20 features, the weights take 19"):
        api.fh_gated(x, wg[:, 1:], wu[:, 1:])
    with pytest.raises(ValueError, match="w_gate is"):
        api.fh_gated(x, wg, wu[1:])
    with pytest.raises(TypeError, match="one dtype"):
        api.fh_gated(x, wg.bfloat16(), wu.bfloat16())
    with pytest.raises(TypeError, match="one dtype"):
        api.fh_gated(x, wg, wu, bg.bfloat16())
    with pytest.raises(ValueError, match="activation"):
        api.fh_gated(x, wg, wu, activation="GELU")
    with pytest.raises(ValueError, match="must be contiguous"):
        api.fh_gated(x, wg.t().contiguous().t(), wu)
    with pytest.raises(ValueError, match="dh must"):
        api.fh_gated_backward(dh[:, 1:], x, wg, wu)
    with pytest.raises(ValueError, match="dh must"):
        api.fh_gated_backward(dh.bfloat16(), x, wg, wu)
    with pytest.raises(TypeError, match="out must"):
        api.fh_gated(x, wg, wu, out=torch.empty(6, 10, device="cuda", dtype=torch.bfloat16))
    with pytest.raises(ValueError, match="overlap"):
        api.fh_gated(torch.zeros(20, device="cuda").expand(6, 20), wg, wu)
    with pytest.raises(TypeError, match="unsupported dtype"):
        api.fh_gated(x.half(), wg.half(), wu.half())


# ---- layers ----------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", [(7,), (3, 5), (2, 3, 4)])
def test_layer_is_its_calls(api, layers, dtype, shape):
    torch.manual_seed(0)
    layer = layers.GatedLinear(48, 70, activation="gelu", device="cuda", dtype=DTYPES[dtype])
    x = torch.randn(*shape, 48, device="cuda").to(DTYPES[dtype]).requires_grad_()
    h = layer(x)
    assert h.shape == (*shape, 70) and h.dtype == DTYPES[dtype]
    dh = torch.randn_like(h)
    h.backward(dh)
    m, parts = x.detach().reshape(-1, 48), [p.detach() for p in (layer.gate.weight, layer.up.weight, layer.gate.bias, layer.up.bias)]
    assert torch.equal(h.detach().reshape(-1, 70), api.fh_gated(m, *parts, "gelu"))
    want = api.fh_gated_backward(dh.reshape(-1, 70), m, *parts, "gelu")
    for got, w in zip((x, layer.gate.weight, layer.up.weight, layer.gate.bias, layer.up.bias), want):
        assert torch.equal(got.grad.reshape(w.shape), w)
    with torch.no_grad():
        assert torch.equal(layer(x), h)


def test_layer_gradients_of_some(layers):
    torch.manual_seed(0)
    layer = layers.GatedLinear(32, 24, device="cuda")
    x = torch.randn(9, 32, device="cuda")
    layer(x).sum().backward()
    whole = layer.up.weight.grad.clone()
    layer.zero_grad()
    layer.gate.weight.requires_grad_(False)
    layer.gate.bias.requires_grad_(False)
    layer(x).sum().backward()
    assert layer.gate.weight.grad is None and layer.gate.bias.grad is None and torch.equal(layer.up.weight.grad, whole)
    shared = layers.gated_linear(x.requires_grad_(), layer.up.weight, layer.up.weight, layer.up.bias, layer.up.bias)
    shared.sum().backward()                                      # the same leaves twice: their gradients add up
    want, _ = torch.autograd.functional.vjp(lambda w: torch.nn.functional.silu(x.detach() @ w.t() + layer.up.bias.detach()) * (x.detach() @ w.t() + layer.up.bias.detach()),
                                            layer.up.weight.detach(), torch.ones(9, 24, device="cuda"))[1], None
    assert torch.allclose(layer.up.weight.grad - whole, want, rtol=1e-4, atol=1e-4)


def test_layer_differentiates_once(layers):
    layer = layers.GatedLinear(16, 8, device="cuda")
    x = torch.randn(4, 16, device="cuda", requires_grad=True)
    (g,) = torch.autograd.grad(layer(x).sum(), x, create_graph=True)
    with pytest.raises(RuntimeError):
        g.sum().backward()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_frozen_layer_and_the_projection_behind_it(api, layers, dtype):
    torch.manual_seed(0)
    layer = layers.GatedLinear(96, 200, activation="gelu_tanh", device="cuda", dtype=DTYPES[dtype])
    down = torch.nn.Linear(200, 96, device="cuda", dtype=DTYPES[dtype])
    x = torch.randn(2, 5, 96, device="cuda").to(DTYPES[dtype])
    layer.freeze()
    stored = api.fh_q8_quantize(down.weight.detach())
    h = layer(x)
    y = layers.q8_linear(h, stored, down.bias)
    assert h.shape == (2, 5, 200) and y.shape == (2, 5, 96) and y.dtype == DTYPES[dtype] and not y.requires_grad

    def product(x, w, bias):
        return R.q8_product(R.stored(x), R.stored(w.detach()), bias.detach())

    m = x.reshape(-1, 96)
    want, bound = R.gated(product(m, layer.gate.weight, layer.gate.bias), product(m, layer.up.weight, layer.up.bias), "gelu_tanh", DTYPES[dtype])
    R.check(h.reshape(-1, 200), want, bound)
    want, bound = product(h.reshape(-1, 200), down.weight, down.bias)
    R.check(y.reshape(-1, 96), want, bound + R.HALF[DTYPES[dtype]] * (want.abs() + bound))
    assert layer.thaw()(x).requires_grad


def test_tangents_are_refused(layers):
    import torch.autograd.forward_ad as fwAD
    layer = layers.GatedLinear(8, 8, device="cuda")
    x = torch.randn(3, 8, device="cuda")
    with fwAD.dual_level():
        dual = fwAD.make_dual(x, torch.ones_like(x))
        with pytest.raises((NotImplementedError, RuntimeError)):
            layer(dual)
        with torch.no_grad(), pytest.raises(NotImplementedError, match="tangent"):
            layer(dual)
        layer.freeze()
        with pytest.raises(NotImplementedError, match="tangent"):
            layer(dual)


def test_training_step_under_saved_activations(api, layers):
    """The input alone is stored compressed; the gradients are those of the call on what was restored, bit for bit."""
    from paper_2510_11400_amd import hooks
    torch.manual_seed(0)
    layer = layers.GatedLinear(64, 128, device="cuda")
    x = torch.randn(8, 64, 64, device="cuda", requires_grad=True)
    saved = hooks.SavedActivations(64, 8, exclude=layer.parameters(), record=True)
    with saved:
        h = layer(x)
    assert len(saved.records) == 1
    dh = torch.randn_like(h)
    h.backward(dh)
    restored = api.fh_decompress(*api.fh_compress(x.detach().view(-1), 64, 8), x.numel(), 64, 8).view(512, 64)
    assert not torch.equal(restored, x.detach().view(512, 64))
    want = api.fh_gated_backward(dh.view(512, 128), restored, *(p.detach() for p in (layer.gate.weight, layer.up.weight, layer.gate.bias, layer.up.bias)))
    for got, w in zip((x, layer.gate.weight, layer.up.weight, layer.gate.bias, layer.up.bias), want):
        assert torch.equal(got.grad.view(w.shape), w)


def test_a_block_of_layers_trains_and_is_served(api, layers):
    """Norm, gated projection and a projection in microscaled form in one step of autograd, each layer's gradients those of its calls; frozen, the
    block replays from a graph as it runs."""
    torch.manual_seed(0)
    gated, down = layers.GatedLinear(64, 96, device="cuda", dtype=torch.bfloat16), torch.nn.Linear(96, 64, device="cuda", dtype=torch.bfloat16)
    norm = layers.LayerNorm(64, device="cuda", dtype=torch.bfloat16)
    x = torch.randn(130, 64, device="cuda").bfloat16().requires_grad_()
    h = gated(norm(x))
    h.retain_grad()
    y = layers.mx_linear(h, down.weight, down.bias)
    y.backward(torch.randn_like(y))
    m = norm(x).detach()
    want = api.fh_gated_backward(h.grad, m, *(p.detach() for p in (gated.gate.weight, gated.up.weight, gated.gate.bias, gated.up.bias)))
    for got, w in zip((gated.gate.weight, gated.up.weight, gated.gate.bias, gated.up.bias), want[1:]):
        assert torch.equal(got.grad, w)
    assert down.weight.grad is not None and bool(torch.isfinite(x.grad).all())

    gated.freeze()
    stored = api.fh_q8_quantize(down.weight.detach())
    token = torch.randn(1, 64, device="cuda").bfloat16()

    def block(t):
        with torch.no_grad():
            return layers.q8_linear(gated(norm(t)), stored, down.bias)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        block(token)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        answer = block(token)
    for i in range(5):
        token.copy_(torch.randn(1, 64, device="cuda"))
        graph.replay()
        assert torch.equal(answer, block(token))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_captured_step(layers, dtype):
    """Forward and backward pass in a graph, replayed on changing inputs with eager work in between."""
    torch.manual_seed(0)
    layer = layers.GatedLinear(100, 70, device="cuda", dtype=DTYPES[dtype])
    x = torch.randn(200, 100, device="cuda").to(DTYPES[dtype]).requires_grad_()
    dh = torch.randn(200, 70, device="cuda").to(DTYPES[dtype])
    leaves = [x, *layer.parameters()]

    def step():
        h = layer(x)
        return [h.detach(), *torch.autograd.grad(h, leaves, dh)]

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        kept = step()
    for i in range(5):
        with torch.no_grad():
            x.copy_(torch.randn(200, 100, device="cuda"))
            dh.copy_(torch.randn(200, 70, device="cuda"))
        graph.replay()
        torch.cuda.synchronize()
        want = step()
        assert all(torch.equal(a, b) for a, b in zip(kept, want))


def test_another_stream(api):
    """With `stream` the work goes there, whatever is current."""
    x, wg, wu, bg, bu, dh = _inputs(300, 128, 96, torch.bfloat16)
    want = api.fh_gated(x, wg, wu, bg, bu), *api.fh_gated_backward(dh, x, wg, wu, bg, bu)
    q = [api.fh_q8_quantize(p) for p in (x, wg, wu)]
    want8 = api.fh_q8_gated(*q, bg, bu)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    got = api.fh_gated(x, wg, wu, bg, bu, stream=side), *api.fh_gated_backward(dh, x, wg, wu, bg, bu, stream=side)
    q = [api.fh_q8_quantize(p, stream=side) for p in (x, wg, wu)]
    got8 = api.fh_q8_gated(*q, bg, bu, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip(got, want)) and torch.equal(got8, want8)


def test_callers_workspaces(api):
    """A workspace of the size that the library names serves, and one that is too small is refused."""
    import ctypes
    x, wg, wu, bg, bu, dh = _inputs(70, 100, 50, torch.float32)

    def layer(backward):
        l = api.fh_gated_layer(70, 100, 50, 0, 0, 3, 0, x.data_ptr(), 100, wg.data_ptr(), 100, wu.data_ptr(), 100, bg.data_ptr(), bu.data_ptr(), None, 50, 0, dh.data_ptr(), 50)
        l.db_gate = l.db_up = 16                                 # not NULL, which is all that is looked at
        return api.raw_library().fh_gated_workspace_bytes(ctypes.byref(l), backward)

    for backward, call in ((0, lambda w: (api.fh_gated(x, wg, wu, bg, bu, workspace=w),)), (1, lambda w: api.fh_gated_backward(dh, x, wg, wu, bg, bu, workspace=w))):
        need = layer(backward)
        want = call(None)
        if not need:
            continue
        room = torch.full((need + 256,), 170, dtype=torch.uint8, device="cuda")
        got = call(room[:need])
        assert all(torch.equal(a, b) for a, b in zip(got, want)) and bool((room[need:] == 170).all())
        with pytest.raises(api.FedHybridError):
            call(room[:need - 1])


def test_the_example_runs_and_its_gradients_are_its_layers(api, layers):
    """Two steps and the served model; a step's gradients are those of the layers' calls on what was restored."""
    import importlib.util
    import math
    import os
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "gated_layers.py")
    spec = importlib.util.spec_from_file_location("gated_layers_example", path)
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    first, last, share = example.main(steps=2, tokens=512, features=64, hidden=96, classes=8)
    assert math.isfinite(first) and math.isfinite(last) and 0.0 <= share <= 1.0
    torch.manual_seed(1)
    model = example.Model(64, 96, 8)
    x = torch.randn(300, 64, device="cuda").bfloat16()
    y = model(x)
    dy = torch.randn_like(y)
    y.backward(dy)
    m = model.norm(x).detach()
    parts = [p.detach() for p in (model.gated.gate.weight, model.gated.up.weight, model.gated.gate.bias, model.gated.up.bias)]
    h = api.fh_gated(m, *parts).requires_grad_()
    layers.mx_linear(h, model.down.weight.detach(), model.down.bias.detach()).backward(dy)
    want = api.fh_gated_backward(h.grad, m, *parts)
    for p, w in zip((model.gated.gate.weight, model.gated.up.weight, model.gated.gate.bias, model.gated.up.bias), want[1:]):
        assert torch.equal(p.grad, w)
