"""Steps of the layers on the GPU: what precision, memory, streams and derivatives they keep to beside their values."""
from __future__ import annotations

import gc

import numpy as np
import pytest

import mx_reference as R

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def layers():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a visible MI355X")
    from paper_2510_11400_amd import layers as _layers
    return _layers


@pytest.fixture(scope="module")
def api(layers):
    return layers.api


def _randn(g, *shape, dtype=torch.bfloat16):
    return torch.randn(*shape, generator=g, device="cuda").to(dtype)


# ---- the gradient of a norm's output stays in fp32 -------------------------------------------------
@pytest.mark.parametrize("tokens, features, out", [(1, 40, 7), (33, 100, 300), (300, 768, 64), (70, 2100, 33), (600, 1500, 40), (20, 5000, 40), (9, 17000, 40)])
@pytest.mark.parametrize("params", [torch.bfloat16, torch.float32])
def test_a_wide_gradient_is_not_rounded_ahead_of_the_norm(api, tokens, features, out, params):
    """The backward half in bf16 with wide_gradient is the product in fp32 and the norm's backward pass of that in fp32, whose dx is
    rounded at the end, bit for bit; where rows are whole and where a norm's kernels of every kind take them."""
    g = torch.Generator(device="cuda").manual_seed(tokens)
    x, dy = _randn(g, tokens, features + 3)[:, 1:1 + features], _randn(g, tokens, out)
    w, b, nw, nb = (_randn(g, *s, dtype=params) for s in ((out, features), (out,), (features,), (features,)))
    _, mean, rstd = api.fh_layer_norm_mx(x, nw, nb, 1e-4, "both")
    dh = api.fh_mx_matmul(api.fh_mx_quantize(dy), api.fh_mx_quantize(w, "columns"), out_dtype=torch.float32)
    dx, dnw, dnb = api.fh_layer_norm_backward(dh, x.float(), mean, rstd, nw.float())
    narrow, layer = api.MxLayer(x, w, b, True, nw, nb, 1e-4), api.MxLayer(x, w, b, True, nw, nb, 1e-4, wide_gradient=True)
    assert torch.equal(layer.forward(), narrow.forward())
    got = layer.backward(dy, x, nw)
    assert torch.equal(got[1], narrow.backward(dy, x, nw)[1])
    layer.needs_weight = False
    for got in (got, layer.backward(dy, x, nw)):
        assert torch.equal(got[0], dx.bfloat16()) and torch.equal(got[2], dnw.to(params)) and torch.equal(got[3], dnb.to(params))


@pytest.mark.parametrize("tokens, features, out", [(130, 300, 130), (512, 768, 260)])
def test_the_steps_input_gradient_is_rounded_once(layers, tokens, features, out):
    """dx of a bf16 step, value by value: the operands' codes are exact, the product is off by its sums' rounding (R.product's bound p), the norm's
    backward pass by R.layer_norm_backward's with the kernel's own statistics; p passes through it as dx itself does, linear in its three terms.
    Then one rounding to bf16, half a step of the value.  (A gradient rounded in between would add 2^-9 of itself on average, which where
    the terms cancel is many steps of dx.)"""
    g = torch.Generator(device="cuda").manual_seed(5)
    x, dy, w, nw, nb = _randn(g, tokens, features), _randn(g, tokens, out), _randn(g, out, features), 1 + 0.2 * _randn(g, features), _randn(g, features)
    leaf = x.clone().requires_grad_()
    dx, = torch.autograd.grad(layers.layer_norm_mx_linear(leaf, nw, nb, w), leaf, dy)
    _, mean, rstd = layers.api.fh_layer_norm_mx(x, nw, nb)
    xm, gm, wm, weight, mean, rstd = (v.double().cpu().numpy() for v in (x, dy, w, nw, mean, rstd))
    blocks = lambda v: R.restored(R.stored(v.astype(np.float32))[0], *v.shape)  # noqa: E731
    dh, p = R.product(blocks(gm), blocks(wm.T))
    want, _, _, bound, _, _ = R.layer_norm_backward(dh, xm, mean, rstd, weight)
    h, pw = (xm - mean[:, None]) * rstd[:, None], p * np.abs(weight)
    bound = bound + np.abs(rstd[:, None]) * (pw + pw.mean(1, keepdims=True) + np.abs(h) * (pw * np.abs(h)).mean(1, keepdims=True))
    far = np.abs(dx.double().cpu().numpy() - want)
    bad = np.argwhere(~(far <= bound + R.HALF_STEP["bf16"] * (np.abs(want) + bound)))
    assert bad.size == 0, f"{len(bad)} of {want.size} off, first at {bad[0]}: {far[tuple(bad[0])]:.3g}"


# ---- what the backward half is given again ------------------------------------------------------------
@pytest.mark.parametrize("params, other", [(torch.float32, torch.bfloat16), (torch.bfloat16, torch.float32)])
def test_the_norms_weight_has_to_be_of_the_parameters_dtype(layers, api, params, other):
    """The kernel reads it by that dtype: twice its bytes where it is the narrower one, other numbers where it is the wider."""
    g = torch.Generator(device="cuda").manual_seed(1)
    x, dy = _randn(g, 64, 300), _randn(g, 64, 40)
    w, nw = _randn(g, 40, 300, dtype=params), _randn(g, 300, dtype=params)
    layer = api.MxLayer(x, w, norm=True, norm_weight=nw)
    layer.forward()
    with pytest.raises(TypeError, match="norm_weight"):
        layer.backward(dy, x, nw.to(other))
    assert layer.backward(dy, x, nw)[0].shape == x.shape
    leaf = x.clone().requires_grad_()                                     # and where a saved-tensor hook gives it back
    with torch.autograd.graph.saved_tensors_hooks(lambda t: t, lambda t: t.to(other) if t.shape == nw.shape else t):
        y = layers.layer_norm_mx_linear(leaf, nw, None, w)
    with pytest.raises(TypeError, match="norm_weight"):
        y.sum().backward()


# ---- streams: whose memory a call takes, shown by addresses, never by what a race would leave -----------
def _busy(stream):
    """Some ten milliseconds of nothing on `stream`."""
    with torch.cuda.stream(stream):
        torch.cuda._sleep(20_000_000)


def _calls(api, g):
    """{name: call(stream) -> its results}, of inputs that every stream may read"""
    x, dy, nw = _randn(g, 608, 704), _randn(g, 608, 704), _randn(g, 704)
    long_a = api.fh_mx_quantize(_randn(g, 96, 40000))
    m = api.fh_mx_quantize(x)
    y, mean, rstd = api.fh_layer_norm(x, nw)
    assert api.mx_matmul_workspace_bytes(96, 96, 40000) > 0
    return {
        "quantize": lambda s: [q.data for q in api.fh_mx_quantize(x, "both", stream=s)],
        "dequantize": lambda s: [api.fh_mx_dequantize(m, stream=s)],
        "matmul": lambda s: [api.fh_mx_matmul(long_a, long_a, stream=s)],
        "layer_norm": lambda s: list(api.fh_layer_norm(x, nw, stream=s)),
        "layer_norm_mx": lambda s: [(r := api.fh_layer_norm_mx(x, nw, stream=s))[0].data, *r[1:]],
        "layer_norm_backward": lambda s: list(api.fh_layer_norm_backward(dy, x, mean, rstd, nw, stream=s)),
    }


def _spans(tensors):
    return [(t.untyped_storage().data_ptr(), t.untyped_storage().data_ptr() + t.untyped_storage().nbytes()) for t in tensors]


def _apart(a, b):
    return all(p[1] <= q[0] or q[1] <= p[0] for p in a for q in b)


def _blocks_like(tensors):
    """Blocks of the same sizes, from the current stream's memory."""
    return [torch.empty(t.untyped_storage().nbytes(), dtype=torch.uint8, device="cuda") for t in tensors]


CALLS = ["quantize", "dequantize", "matmul", "layer_norm", "layer_norm_mx", "layer_norm_backward"]


@pytest.mark.parametrize("name", CALLS)
def test_results_on_another_stream_take_its_memory(api, name):
    """Not blocks that the current stream has just let go and may still read; nor does the current stream get blocks of theirs while the other
    one works; and they stay where they are while the current stream still reads them."""
    call = _calls(api, torch.Generator(device="cuda").manual_seed(2))[name]
    want = [t.clone() for t in call(None)]
    torch.cuda.synchronize()
    here, side = torch.cuda.current_stream(), torch.cuda.Stream()
    freed = _blocks_like(want)
    spans = _spans(freed)
    del freed
    got = call(side)
    assert _apart(_spans(got), spans)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))

    _busy(side)
    got = call(side)
    theirs = _spans(got)
    del got
    mine = _blocks_like(want)
    assert _apart(_spans(mine), theirs)
    torch.cuda.synchronize()
    del mine

    got = call(side)
    side.synchronize()
    _busy(here)
    read = [t.clone() for t in got]                              # behind the current stream's other work
    theirs = _spans(got)
    del got
    again = call(side)
    assert _apart(_spans(again), theirs)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(read, want))


def test_a_workspace_on_another_stream(api):
    """A product whose sum is split, with the current stream's allocations behind it."""
    call = _calls(api, torch.Generator(device="cuda").manual_seed(3))["matmul"]
    want = call(None)[0].clone()
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(3):
        got = call(side)[0]
        for k in range(4):
            torch.empty(api.mx_matmul_workspace_bytes(96, 96, 40000), dtype=torch.uint8, device="cuda").fill_(k)
        side.synchronize()
        torch.cuda.synchronize()
        assert torch.equal(got, want)


def test_what_a_layer_keeps_stays_until_its_stream_is_through(api):
    """A layer dropped behind its backward half on another stream than its forward half's, or on the same: its operands' memory is nobody's
    until that half has run."""
    g = torch.Generator(device="cuda").manual_seed(4)
    x, dy, w = _randn(g, 600, 700), _randn(g, 600, 96), _randn(g, 96, 700)
    first = api.MxLayer(x, w)
    first.forward()
    want = first.backward(dy)[:2]
    torch.cuda.synchronize()
    here, one, two = torch.cuda.current_stream(), torch.cuda.Stream(), torch.cuda.Stream()
    for forward, backward in ((None, one), (one, one), (one, two), (one, None)):
        layer = api.MxLayer(x, w)
        layer.forward(stream=forward)
        torch.cuda.synchronize()
        _busy(backward or here)
        got = layer.backward(dy, stream=backward)[:2]
        kept = [layer.kept]
        size, theirs = kept[0].numel(), _spans(kept)
        del layer, kept
        blocks = []
        for stream in (here, one, two):
            if stream is (backward or here) and stream is (forward or here):
                continue                                         # its own next allocation comes behind that half anyway
            with torch.cuda.stream(stream):
                blocks.append(torch.empty(size, dtype=torch.uint8, device="cuda"))
        assert _apart(_spans(blocks), theirs), (forward, backward)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_a_stream_that_is_the_current_one_changes_nothing(api):
    call = _calls(api, torch.Generator(device="cuda").manual_seed(2))["quantize"]
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        got, want = call(side), call(None)
    assert torch.cuda.current_stream() != side
    with pytest.raises(ValueError):
        api.fh_mx_matmul(api.fh_mx_quantize(torch.zeros(4, 40, device="cuda")), api.fh_mx_quantize(torch.zeros(4, 40, device="cuda")),
                         bias=torch.zeros(3, device="cuda"), stream=side)
    assert torch.cuda.current_stream() == torch.cuda.default_stream()     # also behind a refusal
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))


# ---- what is kept for the backward pass goes with it ------------------------------------------------------
def _held(then):
    """Bytes that `then` leaves allocated, and its result.  A block may be up to 1 MiB larger than what was asked for."""
    gc.collect()
    torch.cuda.synchronize()
    before = torch.cuda.memory_allocated()
    result = then()
    return torch.cuda.memory_allocated() - before, result


@pytest.mark.parametrize("norm", [False, True])
def test_the_backward_pass_frees_what_was_kept(layers, api, norm):
    """Also where the graph outlives it: the output is still there, as a loss is through the next step's forward pass.  Of the step only
    the output and the two gradients are left."""
    g = torch.Generator(device="cuda").manual_seed(1)
    x, w, dy = _randn(g, 16384, 768).requires_grad_(), _randn(g, 768, 768).requires_grad_(), _randn(g, 16384, 768)
    operands = api.mx_bytes(768, 16384) + api.mx_bytes(768, 768)
    held, y = _held(lambda: layers.layer_norm_mx_linear(x, None, None, w) if norm else layers.mx_linear(x, w))
    assert held >= y.nbytes + operands
    left, grads = _held(lambda: torch.autograd.grad(y, (x, w), dy))
    assert held + left <= y.nbytes + sum(v.nbytes for v in grads) + 3 * 2 ** 20 < y.nbytes + sum(v.nbytes for v in grads) + operands
    with pytest.raises(RuntimeError, match="second time"):
        torch.autograd.grad(y, (x, w), dy)


def test_a_retained_graph_keeps_it(layers):
    g = torch.Generator(device="cuda").manual_seed(1)
    x, w, dy = _randn(g, 100, 300).requires_grad_(), _randn(g, 40, 300).requires_grad_(), _randn(g, 100, 40)
    y = layers.layer_norm_mx_linear(x, None, None, w)
    first = torch.autograd.grad(y, (x, w), dy, retain_graph=True)
    assert all(torch.equal(a, b) for a, b in zip(first, torch.autograd.grad(y, (x, w), dy)))


def test_checkpointing_keeps_nothing(layers, api):
    """Recomputed in the backward pass, the operands are not held in between; the gradients are the same."""
    from torch.utils.checkpoint import checkpoint
    g = torch.Generator(device="cuda").manual_seed(1)
    x, w, dy = _randn(g, 16384, 768).requires_grad_(), _randn(g, 768, 768).requires_grad_(), _randn(g, 16384, 768)
    want = torch.autograd.grad(layers.layer_norm_mx_linear(x, None, None, w), (x, w), dy)
    held, y = _held(lambda: checkpoint(layers.layer_norm_mx_linear, x, None, None, w, use_reentrant=False))
    assert held <= y.nbytes + 2 ** 20 < y.nbytes + api.mx_bytes(768, 16384)
    assert all(torch.equal(a, b) for a, b in zip(torch.autograd.grad(y, (x, w), dy), want))


def test_what_was_kept_goes_through_hooks_unchanged(layers):
    """SavedActivations leaves it alone, a hook that moves it away and back may, and one that gives back something else is told so."""
    from paper_2510_11400_amd import hooks
    g = torch.Generator(device="cuda").manual_seed(1)
    x, w, dy = _randn(g, 600, 300).requires_grad_(), _randn(g, 40, 300).requires_grad_(), _randn(g, 600, 40)
    want = torch.autograd.grad(layers.mx_linear(x, w), (x, w), dy)
    for context in (hooks.SavedActivations(64, 4, exclude=(w,)), torch.autograd.graph.save_on_cpu()):
        with context:
            y = layers.mx_linear(x, w)
        assert all(torch.equal(a, b) for a, b in zip(torch.autograd.grad(y, (x, w), dy), want))
    for change, error in ((lambda t: t.float(), ValueError), (lambda t: t.cpu(), ValueError), (lambda t: t[:, :-1], layers.api.FedHybridError)):
        with torch.autograd.graph.saved_tensors_hooks(lambda t: t, change):
            y = layers.mx_linear(x, w)
        with pytest.raises(error):
            torch.autograd.grad(y, (x, w), dy)


# ---- a norm's statistics are not activations -----------------------------------------------------------------
@pytest.mark.parametrize("rows", [100, 5000])
def test_the_statistics_stay_exact_under_saved_activations(layers, rows):
    """Rows whose widths differ by 2^24, x itself kept as it is: the gradients are those of an uncompressed step, bit for bit, however many
    rows there are."""
    from paper_2510_11400_amd import hooks
    g = torch.Generator(device="cuda").manual_seed(1)
    width = torch.exp2(torch.randint(-12, 13, (rows, 1), generator=g, device="cuda").float())
    x = (torch.randn(rows, 40, generator=g, device="cuda") * width).requires_grad_()
    w, b = torch.randn(40, generator=g, device="cuda").requires_grad_(), torch.randn(40, generator=g, device="cuda").requires_grad_()
    dy = torch.randn(rows, 40, generator=g, device="cuda")
    want = torch.autograd.grad(layers.layer_norm(x, w, b), (x, w, b), dy)
    with hooks.SavedActivations(256, 4, exclude=(x, w, b)):
        y = layers.layer_norm(x, w, b)
    assert all(torch.equal(p, q) for p, q in zip(torch.autograd.grad(y, (x, w, b), dy), want))
    empty = layers.layer_norm(x[:0], w, b)
    assert not torch.autograd.grad(empty, w, dy[:0])[0].any()


def test_the_gradient_of_a_norms_bias_without_a_weight(layers, api):
    """It is of the bias's dtype, summed in fp32 and not rounded to x's on the way: equal to the sum that the call gives in fp32."""
    g = torch.Generator(device="cuda").manual_seed(1)
    x, dy, b = _randn(g, 300, 70), _randn(g, 300, 70), torch.zeros(70, device="cuda", requires_grad=True)
    db, = torch.autograd.grad(layers.layer_norm(x, None, b), b, dy)
    exact = dy.double().sum(0)
    # 300 terms in a tree and one join: R.layer_norm_backward's depth
    assert db.dtype == torch.float32 and bool(((db.double() - exact).abs() <= (300 / 256 + 300) * R.U32 * dy.double().abs().sum(0)).all())
    assert bool((db.double() - db.bfloat16().double()).any())             # sums that bf16 does not hold
    _, mean, rstd = api.fh_layer_norm(x)
    for dtype in (torch.float32, torch.bfloat16):
        got = api.fh_layer_norm_backward(dy, x, mean, rstd, sums_dtype=dtype)
        assert got[1].dtype == got[2].dtype == dtype and torch.equal(got[2], db.to(dtype))
    assert api.fh_layer_norm_backward(dy, x, mean, rstd)[2].dtype == x.dtype
    with pytest.raises(TypeError, match="weight"):
        api.fh_layer_norm_backward(dy, x, mean, rstd, torch.ones(70, device="cuda"), sums_dtype=torch.bfloat16)
    with pytest.raises(TypeError):
        api.fh_layer_norm_backward(dy, x, mean, rstd, sums_dtype=torch.float16)


@pytest.mark.parametrize("norm", [False, True])
def test_a_layer_keeps_what_its_gradients_need(layers, api, norm):
    """And gives the same ones: for the input alone, for the weight alone, for neither."""
    g = torch.Generator(device="cuda").manual_seed(1)
    x, dy, w, nw = _randn(g, 700, 300), _randn(g, 700, 130), _randn(g, 130, 300), _randn(g, 300)
    given = dict(norm=norm, norm_weight=nw if norm else None)
    again = (x, nw) if norm else ()
    both = api.MxLayer(x, w, **given)
    y = both.forward()
    want = both.backward(dy, *again)
    x_bytes, w_bytes = api.mx_bytes(300, 700), api.mx_bytes(300, 130)
    slack = 2 * 700 * 4 + 1024
    for needs_input, needs_weight, most in ((True, False, w_bytes), (False, True, x_bytes), (True, True, x_bytes + w_bytes)):
        layer = api.MxLayer(x, w, needs_input=needs_input, needs_weight=needs_weight, **given)
        assert torch.equal(layer.forward(), y) and most <= layer.kept.numel() < most + slack
        got = layer.backward(dy, *again)
        for needed, a, b in zip((needs_input, needs_weight, needs_input, needs_input), got, want):
            assert (a is None) if not needed or b is None else torch.equal(a, b)
        layer.needs_input = layer.needs_weight = True
        if not (needs_input and needs_weight):
            with pytest.raises(api.FedHybridError):
                layer.backward(dy, *again)
    none = api.MxLayer(x, w, needs_input=False, needs_weight=False, **given)
    assert torch.equal(none.forward(), y) and none.kept is None


@pytest.mark.parametrize("norm", [False, True])
@pytest.mark.parametrize("needed", [(True, False), (False, True), (True, True)])
def test_no_tokens_for_some_gradients(layers, norm, needed):
    x, w = torch.empty(0, 40, device="cuda", requires_grad=needed[0]), torch.randn(7, 40, device="cuda", requires_grad=needed[1])
    y = layers.layer_norm_mx_linear(x, None, None, w) if norm else layers.mx_linear(x, w)
    grads = torch.autograd.grad(y, [t for t, n in zip((x, w), needed) if n], torch.empty(0, 7, device="cuda"))
    assert y.shape == (0, 7) and all(not v.any() for v in grads)


@pytest.mark.parametrize("norm", [False, True])
@pytest.mark.parametrize("tokens, features, out", [(34, 100, 300), (300, 768, 64), (2600, 770, 777)])
def test_the_step_of_autograd_is_the_layers_calls(layers, api, tokens, features, out, norm):
    """Output and every gradient in bf16, bit for bit: with test_the_layer_calls_are_their_parts, and the parts' own bounds, no tolerance is left for what
    lies between.  The last shape goes through the larger kernels of the product."""
    g = torch.Generator(device="cuda").manual_seed(tokens)
    x, dy = _randn(g, 2, tokens // 2, features), _randn(g, 2, tokens // 2, out)
    w, b, nw, nb = (_randn(g, *s) for s in ((out, features), (out,), (features,), (features,)))
    leaves = [v.clone().requires_grad_() for v in ((x, nw, nb, w, b) if norm else (x, w, b))]
    how = dict(rounding="stochastic", seed=5, tensor_id=6)
    y = layers.layer_norm_mx_linear(*leaves, **how) if norm else layers.mx_linear(*leaves, **how)
    got = torch.autograd.grad(y, leaves, dy)
    xm, gm = x.view(-1, features), dy.view(-1, out)
    layer = api.MxLayer(xm, w, b, norm, nw if norm else None, nb if norm else None, wide_gradient=True, **how)
    assert torch.equal(y.view(-1, out), layer.forward())
    dx, dw, dnw, dnb, db = layer.backward(gm, xm if norm else None, nw if norm else None, bias=True)
    want = (dx.view(x.shape), dnw, dnb, dw, db) if norm else (dx.view(x.shape), dw, db)
    assert all(torch.equal(p, q) for p, q in zip(got, want))
