"""8-bit storage, its products and the gated projection where offsets pass 32 bits."""
from __future__ import annotations

import pytest

torch = pytest.importorskip("torch")
import gated_reference as R  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def api():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a visible MI355X")
    from paper_2510_11400_amd import api as _api
    yield _api
    torch.cuda.empty_cache()


def test_a_matrix_of_more_than_4_gib(api):
    """70000 rows of 65536: 4.6 GB of codes, restored to 9.2 GB, and a product with it on either side."""
    rows, cols = 70000, 65536
    some = torch.tensor([0, 1, 32767, 32768, 65535, 65536, 69998, 69999], device="cuda")
    x = torch.empty(rows, cols, device="cuda", dtype=torch.bfloat16).normal_(generator=torch.Generator(device="cuda").manual_seed(1))
    m = api.fh_q8_quantize(x)
    codes, scales = R.stored(x[some])
    at = api.q8_scales_offset(rows, cols)
    assert torch.equal(m.data[:at].view(torch.int8).view(rows, cols)[some].double(), codes)
    assert torch.equal(m.data[at:].view(torch.float32)[some].double(), scales)
    back = api.fh_q8_dequantize(m, torch.bfloat16)
    assert torch.equal(back[some], (codes.float() * scales.float()[:, None]).bfloat16())
    del x, back
    few = api.fh_q8_quantize(torch.randn(20, cols, device="cuda"))
    other = R.taken_apart(few)
    want, bound = R.q8_product((codes, scales), (other[0], other[2]), None)
    R.check(api.fh_q8_matmul(m, few, out_dtype=torch.float32)[some], want, bound + R.HALF[torch.float32] * (want.abs() + bound))
    got = api.fh_q8_matmul(few, m, out_dtype=torch.float32)[:, some]
    R.check(got, want.t(), (bound + R.HALF[torch.float32] * (want.abs() + bound)).t())
    one = api.Q8Matrix(api.fh_q8_quantize(torch.randn(1, cols, device="cuda")).data, 1, cols)
    first = R.taken_apart(one)
    want, bound = R.q8_product((first[0], first[2]), (codes, scales), None)
    R.check(api.fh_q8_matmul(one, m, out_dtype=torch.float32)[:, some], want, bound + R.HALF[torch.float32] * (want.abs() + bound))


def test_outputs_of_more_than_4_gib(api):
    """A product of 300000 x 8200 values."""
    (a, b) = (api.fh_q8_quantize(torch.randn(n, 100, device="cuda")) for n in (300000, 8200))
    ra, rb = R.taken_apart(a), R.taken_apart(b)
    got = api.fh_q8_matmul(a, b)
    some = torch.tensor([0, 131071, 261892, 261893, 299999], device="cuda")
    want, bound = R.q8_product((ra[0][some], ra[2][some]), (rb[0], rb[2]), None)
    R.check(got[some], want, bound + R.HALF[torch.bfloat16] * (want.abs() + bound))


def test_the_most_tokens(api):
    """2^21 tokens of 64 -> 1100 in bf16: a result of 4.6 GB, gradients of the hidden width of 9.7.  dh is zero but for tokens at both ends, so that dW is
    theirs and every other token's dx is zero."""
    t, k, f = 2 ** 21, 64, 1100
    g = torch.Generator(device="cuda").manual_seed(3)
    x = torch.randn(t, k, generator=g, device="cuda").bfloat16()
    wg, wu = ((torch.randn(f, k, generator=g, device="cuda") / 8).bfloat16() for _ in range(2))
    bg, bu = (torch.randn(f, generator=g, device="cuda").bfloat16() for _ in range(2))
    ends = torch.cat((torch.arange(50), torch.arange(t - 50, t))).cuda()
    h = api.fh_gated(x, wg, wu, bg, bu, "silu")
    want, bound = R.gated(R.dense_product(x[ends], wg, bg), R.dense_product(x[ends], wu, bu), "silu", x.dtype)
    R.check(h[ends], want, bound)
    dh = h.zero_()
    dh[ends] = torch.randn(100, f, generator=g, device="cuda").bfloat16()
    got = api.fh_gated_backward(dh, x, wg, wu, bg, bu, "silu")
    wanted = R.gated_backward(dh[ends], x[ends], wg, wu, bg, bu, "silu")
    R.check(got[0][ends], *wanted[0], "dx")
    got[0][ends] = 0.0
    assert not bool(got[0].any())
    for name, y, (w, b) in zip(("dw_gate", "dw_up", "db_gate", "db_up"), got[1:], wanted[1:]):
        R.check(y, w, b, name)                                   # more zeros to add change nothing


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_rows_far_apart(api, dtype):
    """Row strides of 2^31 values."""
    whole = torch.zeros(2 ** 31 + 256, device="cuda", dtype=dtype)
    x = whole.as_strided((2, 100), (2 ** 31, 1))
    x.copy_(torch.randn(2, 100, device="cuda"))
    codes, scales = R.stored(x.contiguous())
    got = R.taken_apart(api.fh_q8_quantize(x))
    assert torch.equal(got[0], codes) and torch.equal(got[2], scales)
    wg, wu = (torch.randn(30, 100, device="cuda").to(dtype) for _ in range(2))
    near = x.contiguous()
    # strides beyond 32 bits have the rows laid out first, and another kernel than near rows', which adds in another order: (k + 2) 2^-23 of the magnitudes
    # bounds a sum in any order, so both are held to it, and each to itself
    want, bound = R.gated(R.dense_product(near, wg, None), R.dense_product(near, wu, None), "silu", dtype)
    apart = api.fh_gated(x, wg, wu)
    R.check(apart, want, bound)
    R.check(api.fh_gated(near, wg, wu), want, bound)
    far = whole.as_strided((2, 30), (2 ** 31, 1), 128)
    api.fh_gated(x, wg, wu, out=far)
    assert torch.equal(far, apart)
    dh = far.contiguous()
    for a, b in zip(api.fh_gated_backward(far, x, wg, wu), api.fh_gated_backward(dh, near, wg, wu)):
        assert (a is None) == (b is None) and (a is None or torch.equal(a, b))
