"""8-bit integer storage and its products on the GPU.  What is stored is defined exactly and has to be equal; products stay within their
roundings (gated_reference)."""
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


def _values(rows, cols, seed, dtype=torch.float32):
    """Rows of many sizes, some of zeros, values on and beside halves of a step."""
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((rows, cols), generator=g)
    x = torch.where(torch.rand((rows, cols), generator=g) < 0.2, torch.randint(-127, 128, (rows, cols), generator=g) / 64.0 + 0.0078125, x)
    x = x * torch.exp2(torch.randint(-12, 12, (rows, 1), generator=g).float())
    x[torch.rand(rows, generator=g) < 0.05] = 0.0
    return x.to(dtype).cuda()


def _check_stored(api, x):
    m = api.fh_q8_quantize(x)
    assert (m.rows, m.cols) == tuple(x.shape) and m.nbytes == api.q8_bytes(*x.shape)
    if m.nbytes == 0:
        return m
    codes, scales = R.stored(x)
    got, rest, got_scales = R.taken_apart(m)
    assert torch.equal(got, codes), f"{int((got != codes).sum())} codes differ"
    assert not rest.any(), "the padding is not zero"
    assert torch.equal(got_scales.nan_to_num(nan=-1.0), scales.nan_to_num(nan=-1.0))
    return m


SHAPES = [(0, 5), (1, 1), (1, 127), (1, 4096), (2, 129), (3, 512), (5, 513), (7, 1000), (33, 1024), (64, 1025), (300, 768), (9, 2048), (4, 2049), (3, 4097), (2, 8192),
          (3, 8193), (2, 16384), (2, 16385), (2, 50000), (1030, 33)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows, cols", SHAPES)
def test_stored_and_restored(api, rows, cols, dtype):
    x = _values(rows, cols, rows + cols, DTYPES[dtype])
    m = _check_stored(api, x)
    if rows == 0:
        return
    codes, scales = R.stored(x)
    for out in DTYPES.values():
        back = api.fh_q8_dequantize(m, out)
        assert torch.equal(back, (codes.float() * scales.float()[:, None]).to(out))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_strided_and_unaligned_rows(api, dtype):
    x = _values(70, 400, 1, DTYPES[dtype])
    for part in (x[:, 1:301], x[:, 3:67], x[5:40, 7:200], x.reshape(-1)[3:3 + 20 * 100].view(20, 100), x[::2], x[:1, 5:], x[3:4].expand(1, 400)):
        m = _check_stored(api, part)
        out = torch.full((part.shape[0], part.shape[1] + 9), 7.0, device="cuda", dtype=DTYPES[dtype])
        api.fh_q8_dequantize(m, out=out[:, 4:4 + part.shape[1]])
        assert torch.equal(out[:, 4:4 + part.shape[1]], api.fh_q8_dequantize(m, DTYPES[dtype]))
        assert bool((out[:, :4] == 7.0).all()) and bool((out[:, 4 + part.shape[1]:] == 7.0).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("cols", [200, 1500, 3000, 20000])
def test_special_values(api, dtype, cols):
    """Zeros of both signs, subnormal numbers, the least row that has a scale, the largest numbers, NaN and infinities."""
    x = torch.randn((14, cols), generator=torch.Generator().manual_seed(2))
    x[0], x[1] = 0.0, -0.0
    x[2] *= 1e-45
    x[3] = 2.0 ** -100
    x[4] = 2.0 ** -101
    x[5] *= 2.0 ** 120
    x[6] = 3.3e38
    x[7, 3], x[8, cols - 1], x[9, 100] = float("nan"), float("inf"), float("-inf")
    x[10] = float("nan")
    x[11, ::2] = 0.0
    x[12, :] = 0.0
    x[12, cols - 1] = -5.0
    m = _check_stored(api, x.to(DTYPES[dtype]).cuda())
    back = api.fh_q8_dequantize(m)
    assert bool(torch.isnan(back[7:11]).all()) and bool(torch.isfinite(back[11:]).all()) and bool(torch.isfinite(back[:7]).all())


def _pair(api, x):
    m = api.fh_q8_quantize(x)
    codes, _, scales = R.taken_apart(m)
    return m, (codes, scales)


@pytest.mark.parametrize("out", ["f32", "bf16"])
@pytest.mark.parametrize("m, n, k", S.PRODUCTS)
def test_products(api, m, n, k, out):
    (a, ra), (b, rb) = _pair(api, _values(m, k, m + k)), _pair(api, _values(n, k, n * 3 + k))
    for bias in (None, torch.randn(n, device="cuda"), torch.randn(n, device="cuda").bfloat16()):
        y, bound = R.q8_product(ra, rb, bias)
        got = api.fh_q8_matmul(a, b, bias, DTYPES[out])
        R.check(got, y, bound + R.HALF[DTYPES[out]] * (y.abs() + bound), (m, n, k))
        again = api.fh_q8_matmul(a, b, bias, DTYPES[out])
        assert torch.equal(got, again)


def test_products_into_rows_of_a_larger_matrix(api):
    (a, ra), (b, rb) = _pair(api, _values(70, 300, 1)), _pair(api, _values(45, 300, 2))
    for out, whole in (("f32", torch.full((90, 61), 7.0, device="cuda")), ("bf16", torch.full((90, 61), 7.0, device="cuda").bfloat16())):
        y, bound = R.q8_product(ra, rb, None)
        api.fh_q8_matmul(a, b, out=whole[10:80, 3:48])
        R.check(whole[10:80, 3:48], y, bound + R.HALF[DTYPES[out]] * (y.abs() + bound))
        rest = whole.clone()
        rest[10:80, 3:48] = 7.0
        assert bool((rest == 7.0).all())


def test_codes_of_minus_128_and_the_longest_sums(api):
    """A stored matrix that another program made: the sum of 2^17 - 1 products of -128 and -128 is below 2^31."""
    k = 2 ** 17 - 1
    data = torch.full((2 * R.padded(k),), -128, dtype=torch.int8, device="cuda").view(2, -1)
    data[:, k:] = 0
    data[1] = -data[1].clamp(min=-127)
    scales = torch.tensor([1.0, 0.5], device="cuda")
    m = api.Q8Matrix(torch.cat((data.reshape(-1).view(torch.uint8), scales.view(torch.uint8))), 2, k)
    got = api.fh_q8_matmul(m, m, out_dtype=torch.float32)
    want = torch.tensor([[128.0 * 128 * k, -128.0 * 127 * k * 0.5], [-128.0 * 127 * k * 0.5, 127.0 * 127 * k * 0.25]], dtype=torch.float64, device="cuda")
    assert torch.equal(got, want.float())


def test_rows_without_numbers_reach_their_own_outputs_alone(api):
    x, w = _values(40, 200, 1), _values(50, 200, 2)
    x[3, 7], w[11, 199] = float("nan"), float("inf")
    got = api.fh_q8_matmul(api.fh_q8_quantize(x), api.fh_q8_quantize(w), out_dtype=torch.float32)
    want = torch.zeros(40, 50, dtype=torch.bool, device="cuda")
    want[3], want[:, 11] = True, True
    assert torch.equal(torch.isnan(got), want)


def test_no_summed_columns(api):
    empty = [api.Q8Matrix(torch.empty(0, dtype=torch.uint8, device="cuda"), rows, 0) for rows in (5, 7)]
    bias = torch.randn(7, device="cuda")
    assert torch.equal(api.fh_q8_matmul(*empty, out_dtype=torch.float32), torch.zeros(5, 7, device="cuda"))
    assert torch.equal(api.fh_q8_matmul(*empty, bias=bias, out_dtype=torch.float32), bias.expand(5, 7))
    h = api.fh_q8_gated(empty[0], empty[1], empty[1], bias, bias, out_dtype=torch.float32)
    want, bound = R.gated((bias.double().expand(5, 7), torch.zeros(5, 7, device="cuda", dtype=torch.float64)), (bias.double().expand(5, 7), 0.0 * bias.double().expand(5, 7)),
                          "silu", torch.float32)
    R.check(h, want, bound)


@pytest.mark.parametrize("out", ["f32", "bf16"])
@pytest.mark.parametrize("m, n, k", S.GATED)
def test_gated(api, m, n, k, out):
    g = torch.Generator().manual_seed(m + n + k)
    (x, rx), (gate, rg), (up, ru) = _pair(api, _values(m, k, m + k)), *(_pair(api, (torch.randn((n, k), generator=g) / k ** 0.5).cuda()) for _ in range(2))
    for i, act in enumerate(ACTIVATIONS):
        bg, bu = ((None, None), (torch.randn(n, device="cuda"), torch.randn(n, device="cuda")), (None, torch.randn(n, device="cuda").bfloat16()))[i]
        h, bound = R.gated(R.q8_product(rx, rg, bg), R.q8_product(rx, ru, bu), act, DTYPES[out])
        got = api.fh_q8_gated(x, gate, up, bg, bu, act, DTYPES[out])
        R.check(got, h, bound, (m, n, k, act))
        assert torch.equal(got, api.fh_q8_gated(x, gate, up, bg, bu, act, DTYPES[out]))


def test_refused_shapes_and_names(api):
    x, w = api.fh_q8_quantize(_values(4, 40, 1)), api.fh_q8_quantize(_values(6, 41, 2))
    with pytest.raises(ValueError, match="40 columns, b 41"):
        api.fh_q8_matmul(x, w)
    with pytest.raises(ValueError, match="40 features, the weights take 41"):
        api.fh_q8_gated(x, w, w)
    with pytest.raises(ValueError, match="w_gate is"):
        api.fh_q8_gated(x, x, w)
    with pytest.raises(ValueError, match="activation"):
        api.fh_q8_gated(x, x, x, activation="relu")
    with pytest.raises(ValueError, match="b_up must be a vector of 4"):
        api.fh_q8_gated(x, x, x, b_up=torch.zeros(5, device="cuda"))
    with pytest.raises(TypeError, match="different dtypes"):
        api.fh_q8_gated(x, x, x, torch.zeros(4, device="cuda"), torch.zeros(4, device="cuda").bfloat16())
    with pytest.raises(ValueError, match="out is"):
        api.fh_q8_matmul(x, x, out=torch.zeros(4, 5, device="cuda"))
    with pytest.raises(TypeError, match="unsupported dtype"):
        api.fh_q8_quantize(torch.zeros(4, 4, device="cuda", dtype=torch.float16))
    with pytest.raises(api.FedHybridError):
        api.fh_q8_matmul(api.Q8Matrix(x.data[:100], 4, 40), x)
