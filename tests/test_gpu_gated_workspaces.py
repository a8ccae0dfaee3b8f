"""A caller's workspaces for the gated projection and its backward pass: the public calls name their size, the work stays inside of it, and one that is a byte too small is refused."""
from __future__ import annotations

import pytest

torch = pytest.importorskip("torch")

pytestmark = pytest.mark.gpu

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


@pytest.fixture(scope="module")
def api():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a visible MI355X")
    from paper_2510_11400_amd import api as _api
    return _api


def _operands(dtype, tokens, features, hidden):
    g = torch.Generator().manual_seed(tokens + features)
    return [torch.randn(s, generator=g).to(DTYPES[dtype]).cuda() for s in ((tokens, features), (hidden, features), (hidden, features), (hidden,), (hidden,), (tokens, hidden))]


def _serves(api, need, call):
    want = call(None)
    room = torch.full((need + 256,), 170, dtype=torch.uint8, device="cuda")
    assert all(a is b or torch.equal(a, b) for a, b in zip(call(room[:need]), want)) and bool((room[need:] == 170).all())
    assert all(a is b or torch.equal(a, b) for a, b in zip(call(room), want))
    with pytest.raises(api.FedHybridError, match="capacity"):
        call(room[:need - 1])


# rows at no multiple of 16 bytes: all three operands are laid out again; few tokens take theirs as they lie
@pytest.mark.parametrize("dtype, tokens, features, hidden", [("f32", 70, 99, 50), ("bf16", 70, 101, 50), ("bf16", 17, 5, 300), ("f32", 700, 1, 1), ("bf16", 1200, 515, 400)])
def test_the_forward_calls(api, dtype, tokens, features, hidden):
    x, wg, wu, bg, bu, _ = _operands(dtype, tokens, features, hidden)
    need = api.gated_workspace_bytes(x, wg, wu)
    chunk = -(-features * x.element_size() // 128) * 128
    assert need >= (tokens + 2 * hidden) * chunk
    _serves(api, need, lambda w: (api.fh_gated(x, wg, wu, bg, bu, workspace=w),))


@pytest.mark.parametrize("dtype, tokens, features", [("f32", 70, 100), ("bf16", 70, 104), ("f32", 16, 99), ("bf16", 9, 101)])
def test_forward_calls_that_need_none(api, dtype, tokens, features):
    x, wg, wu, bg, bu, _ = _operands(dtype, tokens, features, 50)
    assert api.gated_workspace_bytes(x, wg, wu) == 0
    assert torch.equal(api.fh_gated(x, wg, wu, bg, bu, workspace=torch.empty(16, dtype=torch.uint8, device="cuda")), api.fh_gated(x, wg, wu, bg, bu))


@pytest.mark.parametrize("needs", [dict(), dict(needs_weight=False), dict(needs_input=False), dict(needs_bias=False), dict(needs_input=False, needs_weight=False)])
@pytest.mark.parametrize("dtype, tokens, features, hidden", [("f32", 70, 100, 50), ("bf16", 70, 101, 50), ("bf16", 3000, 64, 300), ("f32", 900, 33, 65)])
def test_the_backward_calls(api, dtype, tokens, features, hidden, needs):
    x, wg, wu, bg, bu, dh = _operands(dtype, tokens, features, hidden)
    for biases in ((bg, bu), (bg, None), (None, None)):
        if needs == dict(needs_input=False, needs_weight=False) and biases == (None, None):
            continue                                             # nothing is asked for: nothing is looked at
        need = api.gated_backward_workspace_bytes(x, wg, wu, *biases, **needs)
        assert need >= tokens * 2 * hidden * x.element_size()
        _serves(api, need, lambda w: api.fh_gated_backward(dh, x, wg, wu, *biases, workspace=w, **needs))


def test_what_the_calls_refuse_has_no_size(api):
    x, wg, wu, bg, bu, _ = _operands("f32", 6, 20, 10)
    for size in (api.gated_workspace_bytes, api.gated_backward_workspace_bytes):
        assert size(x[:0], wg, wu) == 0
        with pytest.raises(ValueError, match="20 features, the weights take 19"):
            size(x, wg[:, 1:], wu[:, 1:])
        with pytest.raises(TypeError, match="one dtype"):
            size(x, wg.bfloat16(), wu.bfloat16())
    with pytest.raises(ValueError, match="must be a vector"):
        api.gated_backward_workspace_bytes(x, wg, wu, bg[1:], bu)
    with pytest.raises(ValueError, match="device memory"):
        api.gated_workspace_bytes(x.cpu(), wg, wu)
