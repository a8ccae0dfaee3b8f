"""A gated projection captured with an input that an eager graph of autograd made: refused, as a captured backward pass would have the default stream wait for the capture."""
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


def test_an_input_that_was_computed_before_the_capture(layers):
    layer = layers.GatedLinear(64, 48, device="cuda", dtype=torch.bfloat16)
    leaf = torch.randn(30, 64, device="cuda").bfloat16().requires_grad_()
    dh = torch.randn(30, 48, device="cuda").bfloat16()
    x = leaf * 2.0
    scaled = layer.up.weight.detach().clone().requires_grad_() * 0.5       # of a leaf of its own: the layer's are part of no graph
    torch.cuda.synchronize()
    with torch.cuda.graph(torch.cuda.CUDAGraph()):
        with pytest.raises(RuntimeError, match="x comes of a graph .* outside of this capture"):
            layer(x)
        with pytest.raises(RuntimeError, match="w_up comes of a graph .* outside of this capture"):
            layers.gated_linear(x.detach(), layer.gate.weight, scaled)
        layer(x.detach())
        with torch.no_grad():
            layer(x)
    torch.cuda.synchronize()
    del x, scaled
    leaves = [leaf, *layer.parameters()]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        h = layer(leaf * 2.0)                                    # computed inside: of the capture's stream
        kept = [h.detach(), *torch.autograd.grad(h, leaves, dh)]
    del h
    for _ in range(3):
        with torch.no_grad():
            leaf.copy_(torch.randn(30, 64, device="cuda"))
        graph.replay()
        torch.cuda.synchronize()
        h = layer(leaf * 2.0)
        want = [h.detach(), *torch.autograd.grad(h, leaves, dh)]
        assert all(torch.equal(a, b) for a, b in zip(kept, want))
        del h


def test_an_input_of_another_stream(layers):
    """What was computed on a stream of its own before the capture is no hindrance outside of one, and eager calls are never refused."""
    layer = layers.GatedLinear(64, 48, device="cuda")
    leaf = torch.randn(30, 64, device="cuda", requires_grad=True)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        x = leaf * 2.0
    torch.cuda.current_stream().wait_stream(side)
    layer(x).sum().backward()
    want = leaf.grad.clone()
    leaf.grad = None
    layer(leaf * 2.0).sum().backward()
    assert torch.equal(leaf.grad, want)
