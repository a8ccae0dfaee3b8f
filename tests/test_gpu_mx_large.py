"""Sizes whose launches pass what one dimension of a launch may have (2^32 threads).  Memory for them is asked for first."""
from __future__ import annotations

import gc

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.fixture
def api():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a visible MI355X")
    from paper_2510_11400_amd import api as _api
    yield _api
    gc.collect()
    torch.cuda.empty_cache()


def _room(gib):
    gc.collect()
    torch.cuda.empty_cache()
    free = torch.cuda.mem_get_info()[0]
    if free < (gib + 16) * 2 ** 30:
        pytest.skip(f"{free / 2 ** 30:.0f} GiB are free, {gib + 16} wanted")


def test_norms_backward_pass_over_very_long_rows(api):
    """One row of 2^27 + 65 columns: more columns than the join of the sums has workgroups for in one dimension.  With one row dbias is dy and
    dweight dy * (x - mean) * rstd, rounded to bf16 from three binary32 operations."""
    _room(8)
    print("[large] norm backward", flush=True)
    cols = 2 ** 27 + 65
    g = torch.Generator(device="cuda").manual_seed(1)
    x, dy = (torch.randn(1, cols, generator=g, device="cuda", dtype=torch.float32).bfloat16() for _ in range(2))
    mean, rstd = torch.full((1,), 0.25, device="cuda"), torch.full((1,), 0.75, device="cuda")
    dx, dw, db = api.fh_layer_norm_backward(dy, x, mean, rstd)
    right = torch.equal(db, dy[0]), torch.equal(dw, (dy[0].float() * ((x[0].float() - 0.25) * 0.75)).bfloat16())
    assert right == (True, True)
    # dx from the sums in binary64, which are small beside dy: a half step of bf16, and of binary32 for what led there
    g64, h = dy[0].double(), (x[0].double() - 0.25) * 0.75
    want = 0.75 * (g64 - g64.mean() - h * (g64 * h).mean())
    # sums of 2^27 terms in a tree of 2^17 a thread and 16 levels, over 2^27: (2^17 + 64) 2^-24 mean|g| and mean|g h| are under 0.008 * 0.8
    far = (dx[0].double() - want).abs()
    right = bool((far <= 2.0 ** -8 * want.abs() + 0.0064 * (1 + h.abs())).all())
    assert right


def test_layer_norm_of_very_many_long_rows(api):
    """2^22 + 3 rows of 16385 columns, in place: a workgroup of 1024 threads a row."""
    _room(140)
    print("[large] layer norm", flush=True)
    rows, cols, tail = 2 ** 22 + 3, 16385, 5
    g = torch.Generator(device="cuda").manual_seed(2)
    last, first = (torch.randn(tail, cols, generator=g, device="cuda").bfloat16() for _ in range(2))
    x = torch.zeros((rows, cols), dtype=torch.bfloat16, device="cuda")
    x[-tail:], x[:tail] = last, first
    y, mean, rstd = api.fh_layer_norm(x, out=x)
    for part, alone in ((slice(-tail, None), last), (slice(None, tail), first)):
        want = api.fh_layer_norm(alone)
        assert torch.equal(y[part], want[0]) and torch.equal(mean[part], want[1]) and torch.equal(rstd[part], want[2])
    assert not mean[tail:-tail].any() and int((y[tail:-tail:4096] != 0).sum()) == 0


def test_codes_of_very_many_narrow_rows(api):
    """2^29 + 5 rows of one fp32 column, stochastically rounded by rows: 2^23 tiles.  Values of the grid stay what they are however they are
    rounded."""
    _room(84)
    print("[large] codes", flush=True)
    rows = 2 ** 29 + 5
    x = torch.ones((rows, 1), device="cuda")
    x[-7:, 0] = torch.tensor([0.0, -4.0, 6.0, 1.5, -0.5, 3.0, 2.0 ** 90], device="cuda")
    m = api.fh_mx_quantize(x, "rows", "stochastic", 3, 4)
    right = torch.equal(api.fh_mx_dequantize(m), x)
    assert right


def test_products_of_very_many_rows(api):
    """2^29 + 33 outputs in one column: of nothing, which is the bias, by a workgroup each 32."""
    _room(4)
    print("[large] product of nothing", flush=True)
    m = 2 ** 29 + 33
    a, b = (api.MxMatrix(torch.empty(0, dtype=torch.uint8, device="cuda"), r, 0) for r in (m, 1))
    out = torch.zeros((m, 1), dtype=torch.bfloat16, device="cuda")
    api.fh_mx_matmul(a, b, torch.tensor([1.5], device="cuda"), out=out)
    right = bool((out == 1.5).all())                             # no comparison that pytest takes apart value by value
    assert right


def test_a_product_of_very_many_rows(api):
    _room(76)
    print("[large] product", flush=True)
    m, k, tail = 2 ** 29 + 33, 32, 70
    data = torch.zeros(api.mx_bytes(m, k), dtype=torch.uint8, device="cuda")
    a = api.MxMatrix(data, m, k)
    g = torch.Generator(device="cuda").manual_seed(5)
    last = api.fh_mx_quantize(torch.randn(tail + 32, k, generator=g, device="cuda"))       # whole groups of scales: rows from a multiple of 32 on
    rows = m - m // 32 * 32 + 64                                                          # the last 65 rows
    codes, scales = api.mx_scales_offset(m, k), api.mx_scales_offset(tail + 32, k)
    data[codes - rows * 128:codes] = last.data[:rows * 128]
    data[codes + (m - rows) // 32 * 256:] = last.data[scales:scales + 3 * 256]
    w = api.fh_mx_quantize(torch.randn(1, k, generator=g, device="cuda"))
    out = api.fh_mx_matmul(a, w)
    want = api.fh_mx_matmul(last, w)
    right = torch.equal(out[-rows:], want[:rows]), not out[:-rows].any()
    assert right == (True, True)


def test_codes_by_rows_of_very_many_rows(api):
    """More rows than one dimension of the grid has workgroups for, and more than one launch has threads for: the values of the grid come back, and
    the bytes are those that the kernel for both forms writes."""
    _room(12)
    print("[large] codes by rows", flush=True)
    g = torch.Generator(device="cuda").manual_seed(6)
    x = torch.randn(600_001, 33, generator=g, device="cuda")
    alone, both = api.fh_mx_quantize(x), api.fh_mx_quantize(x, "both")[0]
    codes = api.mx_scales_offset(*x.shape)
    right = torch.equal(alone.data[:codes + 600_001 // 32 * 256], both.data[:codes + 600_001 // 32 * 256])
    assert right
    del alone, both
    rows = 2 ** 26 + 9
    x = torch.ones((rows, 1), dtype=torch.bfloat16, device="cuda")
    x[-7:, 0] = torch.tensor([0.0, -4.0, 6.0, 1.5, -0.5, 3.0, 2.0 ** 90], device="cuda")
    right = torch.equal(api.fh_mx_dequantize(api.fh_mx_quantize(x), torch.bfloat16), x)
    assert right
