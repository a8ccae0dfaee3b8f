"""Layer norm over more rows than the card holds at a time, at every width from which another kernel takes them: forward dense and into codes, and
backward, against binary64 on the GPU within the bounds of mx_reference (whose formulas these are, in torch)."""
from __future__ import annotations

import pytest

import mx_reference as R

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


@pytest.fixture(scope="module")
def api():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a visible MI355X")
    from paper_2510_11400_amd import api as _api
    return _api


def _x(rows, cols, dtype, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    width = torch.exp2(torch.randint(-6, 6, (rows, 1), generator=g, device="cuda").float())
    return (torch.randn(rows, cols, generator=g, device="cuda") * width + 3 * torch.randn(rows, 1, generator=g, device="cuda")).to(DTYPES[dtype]), g


def _within(got, want, bound, dtype, what):
    far, bound = (got.double() - want).abs(), bound + R.HALF_STEP[dtype] * (want.abs() + bound) + 1e-38
    bad = (~(far <= bound)).nonzero()
    assert bad.numel() == 0, f"{what}: {len(bad)} off, first at {bad[0].tolist()}, last at {bad[-1].tolist()}"


def _moments(x, eps):
    """mean, rstd, d = x - mean, and the bounds of mean, x - mean and rstd (R.layer_norm)"""
    n, u = x.shape[1], R.U32
    depth = 64 + n / 1024
    mean = x.mean(1, keepdim=True)
    d = x - mean
    var = (d * d).mean(1, keepdim=True)
    rstd = (var + eps).rsqrt()
    d_mean = (depth + 1) * u * x.abs().mean(1, keepdim=True)
    d_value = d_mean + u * d.abs()
    d_var = (2 * d.abs() * d_value + d_value ** 2).mean(1, keepdim=True) + (depth + 2) * u * var
    return mean, rstd, d, d_mean, d_value, rstd * (0.5 * d_var / (var + eps) * 1.01 + 4 * u)


# rows past what stays on the card at a time, and odd: workgroups take a second row each, some a third
FORWARD = [(70001, 40), (33001, 100), (17001, 250), (8301, 511), (5201, 1000), (4201, 1500), (3301, 2000), (2101, 2049), (4301, 2560), (2101, 2561), (2101, 3071),
           (1601, 3073), (1601, 4096), (1101, 4097), (1101, 6144), (801, 6145), (801, 8192), (1101, 8193), (521, 12288), (521, 12289), (301, 16384), (257, 2300)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows, cols", FORWARD)
def test_forward_of_many_rows(api, rows, cols, dtype):
    print(f"[norm] {rows} {cols} {dtype}", flush=True)
    x, g = _x(rows, cols + 3, dtype, cols)
    x = x[:, 1:1 + cols]
    w, b = (torch.randn(cols, generator=g, device="cuda") for _ in range(2))
    y, mean, rstd = api.fh_layer_norm(x, w, b, 1e-5)
    want_mean, want_rstd, d, d_mean, d_value, d_rstd = _moments(x.double(), 1e-5)
    _within(mean, want_mean[:, 0], d_mean[:, 0], "f32", "mean")
    _within(rstd, want_rstd[:, 0], d_rstd[:, 0], "f32", "rstd")
    h = d * want_rstd
    want = h * w.double() + b.double()
    d_y = w.double().abs() * (d_value * want_rstd + d.abs() * d_rstd + R.U32 * h.abs()) * 1.01 + 2 * R.U32 * (want.abs() + b.double().abs())
    _within(y, want, d_y, dtype, "y")
    for part in (slice(0, 1), slice(rows - 2, rows)):                     # in place, and again
        again = x.contiguous()
        assert torch.equal(api.fh_layer_norm(again, w, b, 1e-5, out=again)[0][part], y[part])


def _values_of(x, mean, rstd, w, b):
    """y in fp32 as the definition has it, from given statistics: exact but for the roundings it names.  w is a power of two and b 1/4, so that the sum
    of the fused step is exact in binary64 and rounded once."""
    h = (x.float() - mean[:, None]) * rstd[:, None]
    return h if w is None else (h.double() * w.double() + b.double()).float()


CODES = [(70001, 40), (9001, 250), (8301, 511), (5201, 1000), (4201, 1500), (3301, 2000), (4301, 2049), (4301, 2304), (4301, 2560), (4301, 2561), (4301, 3071), (1601, 3073),
         (1601, 4096), (1101, 4097), (1101, 6145), (801, 8192), (521, 12289), (301, 16384), (257, 2100), (1536, 2300), (1536, 2900)]


@pytest.mark.parametrize("params", [False, True])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows, cols", CODES)
def test_codes_of_many_rows(api, rows, cols, dtype, params):
    """The statistics within their bounds, and every code and scale that of the value from these statistics."""
    print(f"[norm to codes] {rows} {cols} {dtype} {params}", flush=True)
    x, g = _x(rows, cols, dtype, cols + 1)
    w, b = (torch.exp2(torch.randint(-2, 3, (cols,), generator=g, device="cuda").float()), torch.full((cols,), 0.25, device="cuda")) if params else (None, None)
    want_mean, want_rstd, _, d_mean, _, d_rstd = _moments(x.double(), 1e-5)
    for forms in ("rows", "both"):
        got, mean, rstd = api.fh_layer_norm_mx(x, w, b, 1e-5, forms)
        _within(mean, want_mean[:, 0], d_mean[:, 0], "f32", "mean")
        _within(rstd, want_rstd[:, 0], d_rstd[:, 0], "f32", "rstd")
        want = api.fh_mx_quantize(_values_of(x, mean, rstd, w, b), forms)
        for a, c in zip(*((v if forms == "both" else (v,)) for v in (got, want))):
            codes = api.mx_scales_offset(a.rows, a.cols)
            whole = codes + a.rows // 32 * (-(-a.cols // 256)) * 256      # behind: the scales of a last group, some of rows that do not exist
            assert torch.equal(a.data[:whole], c.data[:whole])
            assert torch.equal(api.fh_mx_dequantize(a), api.fh_mx_dequantize(c))


BACKWARD = [(20001, 40), (9001, 100), (5001, 200), (5001, 500), (5001, 700), (4001, 1000), (3001, 1300), (3001, 2000), (1001, 4000), (601, 8000), (601, 12000), (601, 16000)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows, cols", BACKWARD)
def test_backward_of_many_rows(api, rows, cols, dtype):
    print(f"[norm backward] {rows} {cols} {dtype}", flush=True)
    x, g = _x(rows, cols, dtype, cols + 2)
    dy = torch.randn(rows, cols, generator=g, device="cuda").to(DTYPES[dtype])
    w = 1 + 0.3 * torch.randn(cols, generator=g, device="cuda")
    mean, rstd = x.double().mean(1).float(), (x.double().var(1, unbiased=False) + 1e-5).rsqrt().float()
    dx, dw, db = api.fh_layer_norm_backward(dy, x, mean, rstd, w)
    u, depth, depth_rows = R.U32, 64 + cols / 1024, rows / 256 + 300
    r = rstd.double()[:, None]
    h, gw = (x.double() - mean.double()[:, None]) * r, dy.double() * w.double()
    s1, s2 = gw.mean(1, keepdim=True), (gw * h).mean(1, keepdim=True)
    want = r * (gw - s1 - h * s2)
    d_s1 = (depth + 3) * u * gw.abs().mean(1, keepdim=True)
    d_s2 = (depth + 6) * u * (gw * h).abs().mean(1, keepdim=True)
    _within(dx, want, r * (d_s1 + h.abs() * d_s2 + 6 * u * (gw.abs() + s1.abs() + (h * s2).abs())) * 1.01, dtype, "dx")
    _within(dw, (dy.double() * h).sum(0), (depth_rows + 3) * u * (dy.double() * h).abs().sum(0), "f32", "dweight")
    _within(db, dy.double().sum(0), depth_rows * u * dy.double().abs().sum(0), "f32", "dbias")


@pytest.mark.parametrize("tokens, features", [(20001, 40), (9001, 100), (5001, 200), (5001, 500), (5001, 700), (4001, 1000), (3001, 1300), (3001, 2000), (1001, 4000), (601, 9000)])
def test_a_wide_gradient_over_many_rows(api, tokens, features):
    """The norm's backward pass of an fp32 gradient beside bf16 rows, as a layer calls it: what the pass over fp32 rows gives, rounded."""
    print(f"[wide] {tokens} {features}", flush=True)
    x, g = _x(tokens, features, "bf16", features)
    w, nw = torch.randn(33, features, generator=g, device="cuda").bfloat16(), torch.randn(features, generator=g, device="cuda").bfloat16()
    dy = torch.randn(tokens, 33, generator=g, device="cuda").bfloat16()
    _, mean, rstd = api.fh_layer_norm_mx(x, nw, None, 1e-5, "both")
    dh = api.fh_mx_matmul(api.fh_mx_quantize(dy), api.fh_mx_quantize(w, "columns"), out_dtype=torch.float32)
    want = api.fh_layer_norm_backward(dh, x.float(), mean, rstd, nw.float())
    layer = api.MxLayer(x, w, norm=True, norm_weight=nw, wide_gradient=True)
    layer.forward()
    got = layer.backward(dy, x, nw)
    assert all(torch.equal(p, q.bfloat16()) for p, q in zip((got[0], got[2], got[3]), want))
