"""The gated projection and the 8-bit products called in unusual ways: the same operand twice, two threads at once, graphs in turn, a graph of autograd
from before a capture."""
from __future__ import annotations

import threading

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


@pytest.fixture(scope="module")
def layers(api):
    from paper_2510_11400_amd import layers as _layers
    return _layers


def _normal(seed, *shapes, dtype=torch.bfloat16):
    g = torch.Generator().manual_seed(seed)
    return [torch.randn(s, generator=g).to(dtype).cuda() for s in shapes]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n, k", [(5, 40), (90, 70), (300, 256), (1100, 520)])
def test_the_same_operand_twice(api, n, k, dtype):
    (w, b, dh) = _normal(0, (n, k), (n,), (n, n), dtype=DTYPES[dtype])
    a = api.fh_q8_quantize(w)
    c = [api.fh_q8_quantize(w.clone()) for _ in range(3)]
    assert torch.equal(api.fh_q8_matmul(a, a, b), api.fh_q8_matmul(c[0], c[1], b.clone()))
    assert torch.equal(api.fh_q8_gated(a, a, a, b, b), api.fh_q8_gated(*c, b.clone(), b.clone()))
    apart = [w.clone() for _ in range(3)] + [b.clone() for _ in range(2)]
    assert torch.equal(api.fh_gated(w, w, w, b, b), api.fh_gated(*apart))
    for got, want in zip(api.fh_gated_backward(dh, w, w, w, b, b), api.fh_gated_backward(dh, *apart)):
        assert torch.equal(got, want)
    square = dh.abs()                                            # the result's gradient is the input too
    for got, want in zip(api.fh_gated_backward(square, square, square, square), api.fh_gated_backward(*(square.clone() for _ in range(4)))):
        assert (got is None) == (want is None) and (got is None or torch.equal(got, want))


def test_batches_that_do_not_lie_in_order(api, layers):
    """A transposed batch, and a result's gradient that is one number for all."""
    (x, wg, wu, bg, bu) = _normal(1, (6, 50, 96), (40, 96), (40, 96), (40,), (40,))
    turned = x.transpose(0, 1).detach().requires_grad_()
    h = layers.gated_linear(turned, wg, wu, bg, bu, "gelu_tanh")
    h.sum().backward()
    flat = x.transpose(0, 1).reshape(-1, 96)
    assert torch.equal(h.reshape(-1, 40), api.fh_gated(flat, wg, wu, bg, bu, "gelu_tanh"))
    dx = api.fh_gated_backward(torch.ones(300, 40, device="cuda", dtype=x.dtype), flat, wg, wu, bg, bu, "gelu_tanh")[0]
    assert torch.equal(turned.grad.reshape(-1, 96), dx)


def test_two_threads_at_once(api):
    """Each on a stream of its own, the same kernels over different operands."""
    sets = [_normal(s, (700 + 60 * s, 384), (260, 384), (260, 384), (260,), (260,), (700 + 60 * s, 260)) for s in range(2)]

    def work(x, wg, wu, bg, bu, dh, stream=None):
        stored = [api.fh_q8_quantize(p, stream=stream) for p in (x, wg, wu)]
        return [api.fh_gated(x, wg, wu, bg, bu, stream=stream), *api.fh_gated_backward(dh, x, wg, wu, bg, bu, stream=stream),
                api.fh_q8_gated(*stored, bg, bu, stream=stream), api.fh_q8_matmul(stored[0], stored[1], stream=stream)]

    want = [work(*s) for s in sets]
    torch.cuda.synchronize()
    got, failed = [None, None], []

    def run(i):
        try:
            stream = torch.cuda.Stream()
            with torch.cuda.stream(stream):
                for _ in range(20):
                    got[i] = work(*sets[i])
            stream.synchronize()
        except BaseException as e:  # noqa: BLE001
            failed.append(e)

    threads = [threading.Thread(target=run, args=(i,)) for i in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not failed, failed
    for g, w in zip(got, want):
        assert all(torch.equal(a, b) for a, b in zip(g, w))


def test_graphs_in_turn(api):
    """Two captured passes in one memory pool, replayed in turn on changing operands with eager work in between."""
    sets = [_normal(s + 5, (65 + 300 * s, 200), (130, 200), (130, 200), (130,), (130,), (65 + 300 * s, 130)) for s in range(2)]

    def work(x, wg, wu, bg, bu, dh):
        stored = [api.fh_q8_quantize(p) for p in (x, wg, wu)]
        return [api.fh_gated(x, wg, wu, bg, bu), *api.fh_gated_backward(dh, x, wg, wu, bg, bu), api.fh_q8_gated(*stored, bg, bu)]

    for s in sets:
        work(*s)
    torch.cuda.synchronize()
    graphs, kept, pool = [], [], torch.cuda.graph_pool_handle()
    for s in sets:
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1], pool=pool):
            kept.append(work(*s))
    for i in range(4):
        for s in sets:
            s[0].copy_(torch.randn(s[0].shape, device="cuda"))
            s[5].copy_(torch.randn(s[5].shape, device="cuda"))
        for which in (0, 1) if i % 2 else (1, 0):
            graphs[which].replay()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(kept[which], work(*sets[which])))


def test_a_capture_beside_a_living_graph_of_autograd(layers):
    """A captured backward pass would have the default stream wait for the captured one: the layer refuses, and takes the capture once that graph is gone."""
    layer = layers.GatedLinear(64, 48, device="cuda", dtype=torch.bfloat16)
    x = torch.randn(30, 64, device="cuda").bfloat16().requires_grad_()
    dh = torch.randn(30, 48, device="cuda").bfloat16()
    leaves = [x, *layer.parameters()]
    alive = layer(x)
    torch.cuda.synchronize()
    with torch.cuda.graph(torch.cuda.CUDAGraph()):
        with pytest.raises(RuntimeError, match="still alive"):
            layer(x)
        with torch.no_grad():
            layer(x)                                             # no gradients: nothing in the way
    torch.cuda.synchronize()
    assert torch.autograd.grad(alive, leaves, dh)[0].shape == x.shape
    del alive
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        h = layer(x)
        twice = layer(x)                                         # nodes of this capture are no hindrance
        kept = [h.detach(), *torch.autograd.grad(h + twice, leaves, dh)]
    del h, twice
    for _ in range(3):
        with torch.no_grad():
            x.copy_(torch.randn(30, 64, device="cuda"))
        graph.replay()
        torch.cuda.synchronize()
        h = layer(x)
        want = [h.detach(), *torch.autograd.grad(h + layer(x), leaves, dh)]
        assert all(torch.equal(a, b) for a, b in zip(kept, want))
        del h
