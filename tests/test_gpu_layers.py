"""The layers on the GPU: values and gradients against the formulas in binary64 on the quantised operands, as they are used
in training, in serving, under saved-tensor compression and captured in a graph."""
from __future__ import annotations

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


def _blocks(v, halves=None):
    """v's values on the grid of its rows' blocks."""
    data, _ = R.stored(v.astype(np.float32), halves)
    return R.restored(data, *v.shape)


def _rel(got, want):
    want = torch.as_tensor(want)
    return float((got.double().cpu() - want).norm() / want.norm())


def _case(tokens, features, out, dtype, seed=0):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(2, tokens // 2, features, generator=g).to(dtype)
    w = (torch.randn(out, features, generator=g) / features ** 0.5).to(dtype)
    b = torch.randn(out, generator=g).to(dtype)
    dy = torch.randn(2, tokens // 2, out, generator=g).to(dtype)
    nw, nb = (1 + 0.2 * torch.randn(features, generator=g)).to(dtype), (0.1 * torch.randn(features, generator=g)).to(dtype)
    return x, nw, nb, w, b, dy


def _leaf(v):
    return v.cuda().requires_grad_()


@pytest.mark.parametrize("rounding", ["nearest", "stochastic"])
@pytest.mark.parametrize("tokens, features, out", [(2, 40, 33), (66, 300, 130), (512, 768, 260)])
def test_linear(layers, tokens, features, out, rounding):
    """fp32 throughout: the quantised operands are exact, so the products are off by their sums' rounding alone."""
    x, _, _, w, b, dy = _case(tokens, features, out, torch.float32)
    xc, wc, bc = _leaf(x), _leaf(w), _leaf(b)
    y = layers.mx_linear(xc, wc, bc, rounding, 9, 4)
    dx, dw, db = torch.autograd.grad(y, (xc, wc, bc), dy.cuda())
    xm, wm, gm = x.reshape(-1, features).numpy(), w.numpy(), dy.reshape(-1, out).numpy()
    h = R.philox_halves(*gm.shape, 9, 4) if rounding == "stochastic" else None
    for got, want in ((y, R.product(_blocks(xm), _blocks(wm), b.double().numpy())),
                      (dx, R.product(_blocks(gm, h), _blocks(wm.T))),
                      (dw, R.product(_blocks(gm.T, None if h is None else h.T), _blocks(xm.T)))):
        far = np.abs(got.detach().double().cpu().numpy().reshape(want[0].shape) - want[0])
        assert (far <= want[1] + R.U32 * np.abs(want[0])).all()
    assert _rel(db, gm.astype(float).sum(0)) < 1e-5


@pytest.mark.parametrize("tokens, features, out", [(2, 40, 33), (130, 300, 130), (512, 768, 260)])
def test_norm_and_linear(layers, tokens, features, out):
    """In bf16: outputs are rounded once (2^-9 of a value on average at most), dx and the norm's gradients carry the data
    gradient's rounding as well, and a norm's output next to a border may take the other code: 0.01 of the norm covers all."""
    x, nw, nb, w, b, dy = _case(tokens, features, out, torch.bfloat16)
    leaves = [_leaf(v) for v in (x, nw, nb, w, b)]
    y = layers.layer_norm_mx_linear(*leaves)
    grads = torch.autograd.grad(y, leaves, dy.cuda())
    xm, wm, gm = x.reshape(-1, features).double().numpy(), w.float().numpy(), dy.reshape(-1, out).float().numpy()
    h, mean, rstd, _, _, _ = R.layer_norm(xm, nw.double().numpy(), nb.double().numpy(), 1e-5)
    dh = _blocks(gm) @ _blocks(wm.T).T
    dx, dnw, dnb, _, _, _ = R.layer_norm_backward(dh, xm, mean, rstd, nw.double().numpy())
    want = [_blocks(h) @ _blocks(wm).T + b.double().numpy(), dx, dnw, dnb, _blocks(gm.T) @ _blocks(h.T).T, gm.astype(float).sum(0)]
    for name, got, ref in zip(("y", "dx", "d norm weight", "d norm bias", "dw", "db"), (y, *grads), want):
        assert got.shape == (y.shape if name == "y" else leaves[("dx", "d norm weight", "d norm bias", "dw", "db").index(name)].shape)
        assert _rel(got.detach().reshape(ref.shape), ref) < 0.01, name


def test_norm_layer_is_the_norm(layers):
    x, nw, nb, _, _, _ = _case(64, 300, 8, torch.float32)
    leaves = [_leaf(v) for v in (x, nw, nb)]
    dy = torch.randn(x.shape, generator=torch.Generator().manual_seed(3))
    y = layers.layer_norm(*leaves)
    grads = torch.autograd.grad(y, leaves, dy.cuda())
    ref = [v.double().requires_grad_() for v in (x, nw, nb)]
    d = ref[0] - ref[0].mean(-1, keepdim=True)
    want = d / (d.square().mean(-1, keepdim=True) + 1e-5).sqrt() * ref[1] + ref[2]
    for got, r in zip((y, *grads), (want, *torch.autograd.grad(want, ref, dy.double()))):
        assert got.shape == r.shape and _rel(got.detach(), r.detach()) < 1e-5


def test_gradients_that_nobody_needs_are_not_made(layers):
    x, nw, nb, w, b, dy = (v.cuda() for v in _case(66, 100, 40, torch.float32))
    full = [v.clone().requires_grad_() for v in (x, nw, nb, w, b)]
    want = torch.autograd.grad(layers.layer_norm_mx_linear(*full), full, dy)
    for needed in ((0,), (3,), (1, 2), (4,), (0, 4), (2, 3)):
        leaves = [v.clone().requires_grad_(i in needed) for i, v in enumerate((x, nw, nb, w, b))]
        got = torch.autograd.grad(layers.layer_norm_mx_linear(*leaves), [leaves[i] for i in needed], dy)
        for i, g in zip(needed, got):
            assert torch.equal(g, want[i]), (needed, i)
    lin = [v.clone().requires_grad_() for v in (x, w)]
    want = torch.autograd.grad(layers.mx_linear(*lin), lin, dy)
    for i in (0, 1):
        leaves = [v.clone().requires_grad_(i == k) for k, v in enumerate((x, w))]
        assert torch.equal(torch.autograd.grad(layers.mx_linear(*leaves), leaves[i], dy)[0], want[i])
    assert not layers.mx_linear(x, w).requires_grad


def test_views_and_expanded_gradients(layers):
    """Inputs whose rows are not next to each other, and the gradient of a sum, which is one value seen everywhere."""
    x, _, _, w, _, _ = _case(64, 100, 40, torch.float32)
    wide = torch.randn(2, 32, 130, device="cuda")
    wide[..., 7:107] = x.cuda()
    got, want = [], []
    for src, keep in ((wide[..., 7:107], got), (x.cuda(), want)):
        leaf = src.detach().requires_grad_() if src.is_contiguous() else src
        wc = _leaf(w)
        y = layers.mx_linear(leaf, wc)
        keep += [y.detach(), *torch.autograd.grad(y.sum(), wc)]
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    t = x.transpose(0, 1).cuda()
    assert torch.equal(layers.mx_linear(t, w.cuda()), layers.mx_linear(x.cuda(), w.cuda()).transpose(0, 1))


def test_a_frozen_layer_answers_as_the_trained_one(layers):
    torch.manual_seed(1)
    layer = layers.LayerNormMxLinear(300, 130, device="cuda", dtype=torch.bfloat16)
    for tokens in (1, 2, 17, 100):
        x = torch.randn(tokens, 300, device="cuda", dtype=torch.bfloat16)
        want = layer(x).detach()
        assert torch.equal(layer.freeze()(x), want)
        one = layer(x[-1:])
        # the same sums of one token alone, in another order: an fp32 sum's rounding may fall to the other side of a bf16 border
        assert float((one.float() - want[-1:].float()).abs().max()) <= 2.0 ** -7 * float(want[-1:].float().abs().max())
        assert layer.thaw()(x).requires_grad


def test_training_reduces_the_loss(layers):
    """A few steps of a two-layer model with stochastically rounded gradients under saved-tensor compression."""
    from paper_2510_11400_amd import hooks
    torch.manual_seed(2)
    model = torch.nn.Sequential(layers.LayerNormMxLinear(256, 512, rounding="stochastic", tensor_id=0, device="cuda", dtype=torch.bfloat16),
                                torch.nn.GELU(),
                                layers.LayerNormMxLinear(512, 64, rounding="stochastic", tensor_id=1, device="cuda", dtype=torch.bfloat16))
    x = torch.randn(1024, 256, device="cuda", dtype=torch.bfloat16)
    target = torch.randn(1024, 64, device="cuda", dtype=torch.bfloat16).float()
    opt = torch.optim.SGD(model.parameters(), lr=0.5)
    losses = []
    for step in range(12):
        with hooks.SavedActivations(64, 8, exclude=model.parameters(), first_tensor_id=10 * step):
            loss = (model(x).float() - target).square().mean()
        opt.zero_grad()
        loss.backward()
        opt.step()
        losses.append(float(loss))
    assert model[0].steps == 12
    assert losses[-1] < losses[0] and all(np.isfinite(losses)), losses


def test_captured_in_a_graph(layers):
    """Forward and backward of the layer recorded once, replayed on new inputs between eager work, each replay against the
    eager result.  The leaves of the graph are its own."""
    x, nw, nb, w, _, dy = (v.cuda() for v in _case(200, 300, 130, torch.bfloat16))

    def step(x, dy, leaves):
        xl = x.detach().requires_grad_()
        y = layers.layer_norm_mx_linear(xl, *leaves)
        return [y.detach(), *torch.autograd.grad(y, [xl, *leaves], dy)]

    static_x, static_dy = x.clone(), dy.clone()
    static = [v.clone().requires_grad_() for v in (nw, nb, w)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(static_x, static_dy, static)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step(static_x, static_dy, static)
    for k in range(4):
        g = torch.Generator(device="cuda").manual_seed(k)
        nx, ndy = (torch.randn(v.shape, generator=g, device="cuda").to(v.dtype) for v in (x, dy))
        static_x.copy_(nx)
        static_dy.copy_(ndy)
        graph.replay()
        got = [v.clone() for v in out]
        want = step(nx, ndy, [v.clone().requires_grad_() for v in (nw, nb, w)])
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want)), k


@pytest.mark.parametrize("dtype, params", [(torch.bfloat16, torch.bfloat16), (torch.bfloat16, torch.float32), (torch.float32, torch.float32)])
@pytest.mark.parametrize("norm", [False, True])
@pytest.mark.parametrize("tokens, features, out", [(1, 40, 7), (33, 100, 300), (300, 768, 64), (70, 2100, 33)])
def test_the_layer_calls_are_their_parts(layers, tokens, features, out, norm, dtype, params):
    """MxLayer's two calls against the calls that they stand for, bit for bit, from rows that are not next to each other."""
    from paper_2510_11400_amd import api
    g = torch.Generator(device="cuda").manual_seed(tokens)
    wide = torch.randn(tokens, features + 9, generator=g, device="cuda").to(dtype)
    x, w = wide[:, 5:5 + features], torch.randn(out, features + 3, generator=g, device="cuda").to(params)[:, :features]
    b, nw, nb = (torch.randn(n, generator=g, device="cuda").to(params) for n in (out, features, features))
    dy = torch.randn(tokens, out + 1, generator=g, device="cuda").to(dtype)[:, 1:]
    if norm:
        (xr, xc), mean, rstd = api.fh_layer_norm_mx(x, nw, nb, 1e-4, "both")
    else:
        xr, xc = api.fh_mx_quantize(x, "both")
    wr, wc = api.fh_mx_quantize(w, "both")
    want = api.fh_mx_matmul(xr, wr, b, dtype)
    gr, gc = api.fh_mx_quantize(dy, "both", "stochastic", 3, 8)
    want_dw = api.fh_mx_matmul(gc, xc, out_dtype=params)
    want_dx = api.fh_mx_matmul(gr, wc, out_dtype=dtype)
    want_nw = want_nb = None
    if norm:
        want_dx, want_nw, want_nb = api.fh_layer_norm_backward(want_dx, x, mean, rstd, nw)
        if params != dtype:
            want_nw, want_nb = want_nw.to(params), want_nb.to(params)
    layer = api.MxLayer(x, w, b, norm, nw if norm else None, nb if norm else None, 1e-4, rounding="stochastic", seed=3, tensor_id=8)
    assert torch.equal(layer.forward(), want)
    for _ in range(2):
        got = layer.backward(dy, x, nw if norm else None)
        assert torch.equal(got[0], want_dx) and torch.equal(got[1], want_dw)
        assert (got[2] is None and got[3] is None) if not norm else torch.equal(got[2], want_nw) and torch.equal(got[3], want_nb)
    alone = api.MxLayer(x, w, b, norm, nw if norm else None, nb if norm else None, 1e-4, needs_input=False, needs_weight=False)
    assert torch.equal(alone.forward(), want)


def test_no_tokens(layers):
    x = torch.empty(0, 40, device="cuda", requires_grad=True)
    w = torch.randn(7, 40, device="cuda", requires_grad=True)
    nw = torch.ones(40, device="cuda", requires_grad=True)
    y = layers.layer_norm_mx_linear(x, nw, None, w)
    assert y.shape == (0, 7)
    dx, dnw, dw = torch.autograd.grad(y, (x, nw, w), torch.empty(0, 7, device="cuda"))
    assert dx.shape == (0, 40) and not dnw.any() and not dw.any()


def test_gradients_that_are_one_row_everywhere(layers):
    """The gradient of a sum over tokens reaches the layer as one row expanded over all of them."""
    x, nw, nb, w, _, _ = (v.cuda() for v in _case(64, 100, 40, torch.float32))
    leaves = [v.clone().requires_grad_() for v in (x, nw, nb, w)]
    scale = torch.randn(40, device="cuda")
    y = layers.layer_norm_mx_linear(*leaves)
    got = torch.autograd.grad((y.sum((0, 1)) * scale).sum(), leaves, retain_graph=True)
    want = torch.autograd.grad(y, leaves, scale.expand(y.shape).contiguous())
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    z = [v.clone().requires_grad_() for v in (x.view(64, 100), nw, nb)]
    y = layers.layer_norm(*z)
    got = torch.autograd.grad((y.sum(0) * scale[0]).sum(), z, retain_graph=True)
    want = torch.autograd.grad(y, z, scale[0].expand(y.shape).contiguous())
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_differentiated_once(layers):
    """A second derivative is refused when it is asked for, also where the first one was asked for with a graph."""
    x, w = torch.randn(64, 96, device="cuda").requires_grad_(), torch.randn(40, 96, device="cuda").requires_grad_()
    dy = torch.randn(64, 40, device="cuda").requires_grad_()
    dx, dw = torch.autograd.grad(layers.mx_linear(x, w), (x, w), dy, create_graph=True)
    want = torch.autograd.grad(layers.mx_linear(x, w), (x, w), dy.detach())
    assert torch.equal(dx, want[0]) and torch.equal(dw, want[1])
    with pytest.raises(RuntimeError):
        torch.autograd.grad(dx.sum() + dw.sum(), dy, retain_graph=True)
    with pytest.raises(RuntimeError, match="once"):
        (dx.sum() + dw.sum()).backward()


def test_one_row_as_a_vector_and_no_gradients_without_a_graph(layers):
    x, w, b = torch.randn(96, device="cuda"), torch.randn(40, 96, device="cuda").requires_grad_(), torch.randn(40, device="cuda")
    y = layers.mx_linear(x, w, b)
    assert y.shape == (40,) and y.requires_grad
    with torch.no_grad():
        z = layers.mx_linear(x, w, b)
    assert not z.requires_grad and torch.equal(z, y)
    with torch.inference_mode():
        z = layers.layer_norm_mx_linear(x[None], None, None, w)
    assert z.shape == (1, 40) and torch.equal(z, layers.layer_norm_mx_linear(x[None], None, None, w))


def test_faults_of_a_backward_pass_reach_the_caller(layers):
    """What a saved-tensor hook gives back is checked on autograd's own thread."""
    x, w = torch.randn(64, 96, device="cuda").requires_grad_(), torch.randn(40, 96, device="cuda")
    with torch.autograd.graph.saved_tensors_hooks(lambda t: t, lambda t: t[:, :-1]):
        y = layers.layer_norm_mx_linear(x, None, None, w)
    with pytest.raises(ValueError, match="shape"):
        y.sum().backward()
    with pytest.raises(KeyError):
        layers.mx_linear(x, w, rounding="up")
    with pytest.raises(ValueError):
        layers.mx_linear(x.cpu(), w)
    with pytest.raises(ValueError):
        layers.mx_linear(x, w[:, :-1].contiguous())
    with pytest.raises(TypeError):
        layers.mx_linear(x, w, torch.zeros(40, device="cuda", dtype=torch.bfloat16))


@pytest.mark.parametrize("rounding", ["nearest", "stochastic"])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("tokens, out", [(1, 7), (33, 300), (257, 64), (1030, 129), (70000, 40)])
def test_the_sum_of_the_gradients_rows(layers, tokens, out, dtype, rounding):
    """The bias's gradient beside every choice of the others, against binary64: a value passes 8 + 2 additions in its
    lane, 8 over the waves, 4 + 2 in the join (two runs of 256 tiles at most) and 16 over its waves: 40, each off by 2^-24 of sums that
    the magnitudes' sum bounds; then one rounding to the dtype."""
    from paper_2510_11400_amd import api
    g = torch.Generator(device="cuda").manual_seed(tokens)
    x, w, b = torch.randn(tokens, 40, generator=g, device="cuda").to(dtype), torch.randn(out, 40, generator=g, device="cuda").to(dtype), torch.zeros(out, device="cuda", dtype=dtype)
    dy = torch.randn(tokens, out + 3, generator=g, device="cuda").to(dtype)[:, 1:out + 1]
    exact, size = dy.double().sum(0), dy.double().abs().sum(0)
    limit = 40 * 2.0 ** -24 * size + torch.finfo(dtype).eps / 2 * exact.abs() + 1e-30
    seen = []
    for needs in ((True, True), (True, False), (False, True), (False, False)):
        layer = api.MxLayer(x, w, b, needs_input=needs[0], needs_weight=needs[1], rounding=rounding, seed=1, tensor_id=2)
        layer.forward()
        without = layer.backward(dy)
        *rest, db = layer.backward(dy, bias=True)
        for p, q in zip(rest, without):
            assert (p is None) == (q is None) and (p is None or torch.equal(p, q))
        assert db.dtype == dtype and bool(((db.double() - exact).abs() <= limit).all())
        seen.append(db)
    assert all(torch.equal(seen[0], v) for v in seen[1:])


def test_the_sum_of_no_rows_and_of_broken_ones(layers):
    x, w, b = torch.empty(0, 40, device="cuda"), torch.randn(7, 40, device="cuda"), torch.zeros(7, device="cuda", requires_grad=True)
    db, = torch.autograd.grad(layers.mx_linear(x, w, b), b, torch.empty(0, 7, device="cuda"))
    assert db.shape == (7,) and not db.any()
    x, dy = torch.randn(300, 40, device="cuda"), torch.randn(300, 7, device="cuda")
    dy[299, 2], dy[5, 4] = float("nan"), float("inf")
    db, = torch.autograd.grad(layers.mx_linear(x, w, b), b, dy)
    assert torch.isnan(db[2]) and torch.isinf(db[4]) and torch.isfinite(db[[0, 1, 3, 5, 6]]).all()


def test_a_layer_with_a_bias_captured_in_a_graph(layers):
    """As test_captured_in_a_graph, with the gradient of the linear layer's bias, over more rows than a tile has."""
    x, nw, nb, w, b, dy = (v.cuda() for v in _case(2100, 300, 130, torch.bfloat16))

    def step(x, dy, leaves):
        xl = x.detach().requires_grad_()
        y = layers.layer_norm_mx_linear(xl, *leaves, rounding="stochastic", seed=5)
        return [y.detach(), *torch.autograd.grad(y, [xl, *leaves], dy)]

    static_x, static_dy = x.clone(), dy.clone()
    static = [v.clone().requires_grad_() for v in (nw, nb, w, b)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(static_x, static_dy, static)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step(static_x, static_dy, static)
    for k in range(4):
        g = torch.Generator(device="cuda").manual_seed(k)
        nx, ndy = (torch.randn(v.shape, generator=g, device="cuda").to(v.dtype) for v in (x, dy))
        static_x.copy_(nx)
        static_dy.copy_(ndy)
        graph.replay()
        got = [v.clone() for v in out]
        want = step(nx, ndy, [v.clone().requires_grad_() for v in (nw, nb, w, b)])
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(got, want)), k


def test_the_example_trains_and_serves():
    """16 classes in 256 features, centres 22 apart at noise 2: all but separable, and 1 in 16 right by chance."""
    import importlib.util
    import os
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "microscaled_layers.py")
    spec = importlib.util.spec_from_file_location("microscaled_layers", path)
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    first, last, share = example.main(steps=30)
    assert last < first / 2 and share > 0.5, (first, last, share)
