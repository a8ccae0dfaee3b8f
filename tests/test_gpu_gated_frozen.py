"""A gated projection one of whose weights is frozen: the other's gradient is the same and holds no more memory than its own."""
from __future__ import annotations

import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


@pytest.fixture(scope="module")
def layers():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a visible MI355X")
    from paper_2510_11400_amd import layers as _layers
    return _layers


# the weights' gradients by one part and by several, at sizes whose bytes are multiples of the allocator's and not
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("tokens, features, hidden", [(9, 32, 24), (3000, 64, 300), (700, 515, 257)])
@pytest.mark.parametrize("frozen", ["gate", "up"])
def test_the_other_weights_gradient(layers, frozen, tokens, features, hidden, dtype):
    torch.manual_seed(0)
    layer = layers.GatedLinear(features, hidden, device="cuda", dtype=DTYPES[dtype])
    x = torch.randn(tokens, features, device="cuda").to(DTYPES[dtype])
    dh = torch.randn(tokens, hidden, device="cuda").to(DTYPES[dtype])
    layer(x).backward(dh)
    kept = layer.up if frozen == "gate" else layer.gate
    want = kept.weight.grad.clone()
    layer.zero_grad()
    getattr(layer, frozen).weight.requires_grad_(False)
    layer(x).backward(dh)
    assert getattr(layer, frozen).weight.grad is None and torch.equal(kept.weight.grad, want)
    assert kept.weight.grad.untyped_storage().nbytes() == want.numel() * want.element_size()
