"""Layers whose gradients have no derivatives of their own: a loss with such a gradient in it is refused, whether or not the result's gradient
itself wants one.  Without the refusal the term is dropped and the sum trains without it."""
from __future__ import annotations

import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def layers():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a visible MI355X")
    from paper_2510_11400_amd import layers as _layers
    return _layers


def _gated(layers):
    layer = layers.GatedLinear(16, 8, device="cuda")
    return layer, (layer.gate.weight, layer.up.weight, layer.gate.bias, layer.up.bias)


def _microscaled(layers):
    layer = torch.nn.Linear(16, 8, device="cuda")
    layer.forward = lambda x: layers.mx_linear(x, layer.weight, layer.bias)
    return layer, (layer.weight, layer.bias)


def _norm_microscaled(layers):
    layer = layers.LayerNormMxLinear(16, 8, device="cuda")
    return layer, (layer.norm.weight, layer.norm.bias, layer.linear.weight, layer.linear.bias)


def _norm(layers):
    layer = layers.LayerNorm(16, device="cuda")
    return layer, (layer.weight, layer.bias)


MODULES = {"gated": _gated, "microscaled": _microscaled, "norm and microscaled": _norm_microscaled, "norm": _norm}


def _made(layers, kind):
    """(the module, its leaves: an input of 4 x 16 first)"""
    torch.manual_seed(0)
    module, parameters = MODULES[kind](layers)
    return module, (torch.randn(4, 16, device="cuda", requires_grad=True), *parameters)


@pytest.mark.parametrize("kind", MODULES)
@pytest.mark.parametrize("given", ["sum", "constant", "leaf"])
def test_a_loss_with_a_gradient_in_it(layers, kind, given):
    """dh from a sum, a tensor of its own, and one that wants a gradient."""
    module, leaves = _made(layers, kind)
    h = module(leaves[0])
    dh = torch.randn_like(h).requires_grad_(given == "leaf")
    alone = h.sum() if given == "sum" else h
    plain = torch.autograd.grad(alone, leaves, None if given == "sum" else dh.detach(), retain_graph=True)
    grads = torch.autograd.grad(alone, leaves, None if given == "sum" else dh, create_graph=True)
    for g, p in zip(grads, plain):
        assert torch.equal(g, p) and g.requires_grad and not p.requires_grad
        loss = h.sum() + g.pow(2).sum()
        with pytest.raises(RuntimeError, match="differentiated once"):
            loss.backward(retain_graph=True)
        for leaf in leaves + ((dh,) if given == "leaf" else ()):
            with pytest.raises(RuntimeError, match="differentiated once"):
                torch.autograd.grad(loss, leaf, retain_graph=True)


@pytest.mark.parametrize("kind", MODULES)
def test_behind_other_layers(layers, kind):
    """The input is no leaf and has three dimensions, its rows lie apart: what it was made of is as far from the refusal."""
    module, leaves = _made(layers, kind)
    wide = torch.randn(2, 3, 20, device="cuda", requires_grad=True)
    h = module((wide * 2.0)[..., :16])
    (g,) = torch.autograd.grad(h.sum(), wide, create_graph=True)
    for leaf in (wide, *leaves[1:]):
        with pytest.raises(RuntimeError, match="differentiated once"):
            torch.autograd.grad(h.sum() + g.pow(2).sum(), leaf, retain_graph=True)


@pytest.mark.parametrize("kind", MODULES)
def test_a_step_whose_graph_is_kept(layers, kind):
    """create_graph alone changes nothing: the gradients are the same, the optimiser takes them, and the next step is clean."""
    module, leaves = _made(layers, kind)
    module(leaves[0]).sum().backward()
    want = [leaf.grad.clone() for leaf in leaves]
    for leaf in leaves:
        leaf.grad = None
    module(leaves[0]).sum().backward(create_graph=True)
    assert all(torch.equal(leaf.grad, w) for leaf, w in zip(leaves, want))
    optimiser = torch.optim.SGD(module.parameters(), lr=0.1)
    optimiser.step()
    optimiser.zero_grad()
    module(leaves[0]).sum().backward()
    assert all(bool(torch.isfinite(p.grad).all()) and not p.grad.requires_grad for p in module.parameters())


@pytest.mark.parametrize("kind", MODULES)
def test_one_leaf_alone(layers, kind):
    """Each leaf as the only one that wants a gradient."""
    module, leaves = _made(layers, kind)
    for i in range(len(leaves)):
        for k, leaf in enumerate(leaves):
            leaf.requires_grad_(k == i)
        h = module(leaves[0])
        (g,) = torch.autograd.grad(h.sum(), leaves[i], create_graph=True)
        with pytest.raises(RuntimeError, match="differentiated once"):
            (module(leaves[0]).sum() + g.pow(2).sum()).backward()
