"""Microscaled 4-bit storage and its product on the GPU against binary64.  The stored bytes are defined exactly and have to
be equal; products stay within the rounding of a binary32 sum (mx_reference.product)."""
from __future__ import annotations

import numpy as np
import pytest

import mx_reference as R

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
SEED, TENSOR = 0xFEDCBA9876543210, (3 << 32) + 11


@pytest.fixture(scope="module")
def api():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a visible MI355X")
    from paper_2510_11400_amd import api as _api
    return _api


def _values(rows, cols, seed, dtype="f32"):
    """Rows of many sizes, values on and beside the grid's midpoints, zeros of both signs."""
    rng = np.random.default_rng(seed)
    x = rng.standard_normal((rows, cols)) * np.exp2(rng.integers(-12, 12, (rows, 1)).astype(float))
    grid = rng.choice([0.0, -0.0, 0.25, 0.75, 1.25, 2.5, 5.0, 6.0, 7.99, 0.25000003, -0.75000006], (rows, cols))
    x = np.where(rng.random((rows, cols)) < 0.3, grid, x).astype(np.float32)
    t = torch.from_numpy(x).to(DTYPES[dtype])
    return t, t.float().numpy()


def _check_store(m, want, rows, cols):
    data, known = want
    assert (m.rows, m.cols) == (rows, cols)
    got = m.data.cpu().numpy()
    assert got.size == data.size
    bad = np.flatnonzero((got != data) & known)
    assert bad.size == 0, f"{bad.size} of {data.size} bytes differ, first at {bad[:8]}: {got[bad[:8]]} for {data[bad[:8]]}"


def _check_quantize(api, t, x, forms, rounding):
    rows, cols = x.shape
    halves = R.philox_halves(rows, cols, SEED, TENSOR) if rounding == "stochastic" else None
    kept = api.fh_mx_quantize(t, forms, rounding, SEED, TENSOR)
    kept = kept if forms == "both" else (kept,)
    if forms in ("rows", "both"):
        _check_store(kept[0], R.stored(x, halves), rows, cols)
    if forms in ("columns", "both"):
        _check_store(kept[-1], R.stored(x.T, None if halves is None else halves.T), cols, rows)
    return kept


SHAPES = [(1, 1), (1, 32), (1, 768), (2, 33), (7, 255), (17, 256), (31, 257), (32, 100), (33, 1000), (100, 31), (255, 64), (256, 128),
          (257, 129), (300, 513), (513, 40)]


@pytest.mark.parametrize("rounding", ["nearest", "stochastic"])
@pytest.mark.parametrize("forms", ["rows", "columns", "both"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_stored_bytes(api, dtype, forms, rounding):
    for i, (rows, cols) in enumerate(SHAPES):
        t, x = _values(rows, cols, i, dtype)
        _check_quantize(api, t.cuda(), x, forms, rounding)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_strided_and_unaligned_rows(api, dtype):
    t, x = _values(70, 400, 1, dtype)
    d = t.cuda()
    for at, width in ((1, 300), (3, 64), (8, 257), (5, 33)):
        for forms in ("rows", "both"):
            _check_quantize(api, d[:, at:at + width], x[:, at:at + width], forms, "nearest")
    _check_quantize(api, d[5:40, 7:200], x[5:40, 7:200], "both", "stochastic")
    flat = d.reshape(-1)[3:3 + 20 * 100].view(20, 100)
    _check_quantize(api, flat, x.reshape(-1)[3:3 + 20 * 100].reshape(20, 100), "both", "nearest")


@pytest.mark.parametrize("rounding", ["nearest", "stochastic"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_special_values(api, dtype, rounding):
    """Blocks of zeros, subnormal numbers, the largest and smallest scales, NaN and infinities of both signs."""
    rng = np.random.default_rng(2)
    x = rng.standard_normal((40, 256)).astype(np.float32)
    x[0] = 0.0
    x[1] = -0.0
    x[2] *= np.float32(1e-45)
    x[3] *= np.float32(2.0 ** -127)
    x[4] *= np.float32(2.0 ** -124)
    x[5] *= np.float32(2.0 ** 126)
    x[6, :] = np.float32(3.3e38)
    x[7, 3], x[8, 40], x[9, 255] = np.nan, np.inf, -np.inf
    x[10, :32], x[11, 31] = np.nan, -np.nan
    x[12] = np.float32(2.0 ** -126)
    x[13, ::2] = 0.0
    t = torch.from_numpy(x).to(DTYPES[dtype])
    with np.errstate(over="ignore"):
        _check_quantize(api, t.cuda(), t.float().numpy(), "both", rounding)
        if rounding == "nearest":
            _check_quantize(api, t.cuda(), t.float().numpy(), "rows", rounding)


@pytest.mark.parametrize("out", ["f32", "bf16"])
def test_restored_values(api, out):
    """Every code at every scale byte, 0 and 255 among them."""
    rng = np.random.default_rng(3)
    for rows, cols in ((256, 32), (33, 1), (5, 300), (64, 511), (1, 256)):
        width = R.padded(cols)
        data = rng.integers(0, 256, api.mx_bytes(rows, cols), dtype=np.uint8)
        scales = np.full(data.size - rows * width // 2, 127, np.uint8)
        at = R.scale_positions(rows, width)
        scales[at] = (np.arange(rows)[:, None] + np.arange(width // 32)[None] * 7) % 256
        data[rows * width // 2:] = scales
        m = api.MxMatrix(torch.from_numpy(data).cuda(), rows, cols)
        got = api.fh_mx_dequantize(m, DTYPES[out])
        with np.errstate(over="ignore"):
            want = torch.from_numpy(R.restored(data, rows, cols).astype(np.float32)).to(DTYPES[out])
        assert torch.equal(got.cpu().view(torch.int16 if out == "bf16" else torch.int32)[~want.isnan()],
                           want.view(torch.int16 if out == "bf16" else torch.int32)[~want.isnan()])
        assert torch.equal(got.cpu().isnan(), want.isnan())
        # into a view: its neighbours stay
        wide = torch.full((rows, cols + 7), 5.0, dtype=DTYPES[out], device="cuda")
        api.fh_mx_dequantize(m, out=wide[:, 3:3 + cols])
        assert torch.equal(wide[:, 3:3 + cols].nan_to_num(9.0), got.nan_to_num(9.0))
        assert (wide[:, :3] == 5).all() and (wide[:, 3 + cols:] == 5).all()


def _check_product(api, m, n, k, out, bias_dtype, seed, view=False):
    a, x = _values(m, k, seed)
    b, w = _values(n, k, seed + 1)
    rng = np.random.default_rng(seed)
    bias = None if bias_dtype is None else torch.from_numpy(rng.standard_normal(n).astype(np.float32) * 100).to(DTYPES[bias_dtype])
    qa, qb = api.fh_mx_quantize(a.cuda()), api.fh_mx_quantize(b.cuda())
    va, vb = R.restored(qa.data.cpu().numpy(), m, k), R.restored(qb.data.cpu().numpy(), n, k)
    want, bound = R.product(va, vb, None if bias is None else bias.double().numpy())
    target = None
    if view:
        wide = torch.full((m, n + 9), 3.0, dtype=DTYPES[out], device="cuda")
        target = wide[:, 5:5 + n]
    got = api.fh_mx_matmul(qa, qb, None if bias is None else bias.cuda(), DTYPES[out], out=target)
    if view:
        assert (wide[:, :5] == 3).all() and (wide[:, 5 + n:] == 3).all()
    far = np.abs(got.double().cpu().numpy() - want)
    bound = bound + R.HALF_STEP[out] * (np.abs(want) + bound)
    bad = np.argwhere(~(far <= bound))
    assert bad.size == 0, f"{m} x {n} x {k}: {len(bad)} outputs off, first at {bad[0]}: {far[tuple(bad[0])]} over {bound[tuple(bad[0])]}"
    return qa, qb


PRODUCTS = [(1, 1, 1), (1, 16, 256), (1, 100, 4096), (2, 33, 300), (15, 17, 31), (16, 16, 257), (17, 250, 1000), (33, 64, 2049),
            (64, 65, 512), (65, 300, 777), (100, 128, 3000), (127, 129, 255), (128, 256, 768), (129, 127, 1300), (200, 1000, 1537),
            (256, 256, 256), (257, 511, 513), (300, 33, 5000), (33, 300, 5000), (520, 390, 1024), (1, 3000, 64), (3000, 1, 64),
            (96, 96, 40000), (640, 640, 8200)]


@pytest.mark.parametrize("m, n, k", PRODUCTS)
def test_products(api, m, n, k):
    print(f"[product] {m} {n} {k}", flush=True)
    _check_product(api, m, n, k, "f32", None, m + n)
    _check_product(api, m, n, k, "bf16", "f32", m + n + 1)


@pytest.mark.parametrize("m, n, k", [(1, 70, 300), (40, 130, 513), (260, 300, 1000)])
def test_products_into_views(api, m, n, k):
    _check_product(api, m, n, k, "f32", "bf16", 5, view=True)
    _check_product(api, m, n, k, "bf16", None, 6, view=True)


def test_product_of_nothing_is_the_bias(api):
    a, b = (api.MxMatrix(torch.empty(0, dtype=torch.uint8, device="cuda"), r, 0) for r in (5, 40))
    bias = torch.randn(40, device="cuda")
    for dtype in DTYPES.values():
        got = api.fh_mx_matmul(a, b, bias, dtype)
        assert torch.equal(got, bias.to(dtype).expand(5, 40))
        assert not api.fh_mx_matmul(a, b, None, dtype).any()


def test_broken_blocks_reach_their_rows_alone(api):
    """A block of NaN makes the sums of its row NaN and no others; scale bytes of rows that do not exist are never used."""
    for m, n, k in ((3, 20, 300), (40, 70, 600), (300, 270, 513)):
        a, x = _values(m, k, 1)
        b, w = _values(n, k, 2)
        a[m // 2, k // 3] = float("nan")
        b[n - 1, 0] = float("inf")
        qa, qb = api.fh_mx_quantize(a.cuda()), api.fh_mx_quantize(b.cuda())
        for q, rows in ((qa, m), (qb, n)):
            at = np.setdiff1d(np.arange(q.data.numel() - api.mx_scales_offset(rows, k)), R.scale_positions(rows, R.padded(k)))
            q.data[torch.from_numpy(at).cuda() + api.mx_scales_offset(rows, k)] = 255
        got = api.fh_mx_matmul(qa, qb, out_dtype=torch.float32).cpu()
        want = torch.zeros(m, n, dtype=torch.bool)
        want[m // 2], want[:, n - 1] = True, True
        assert torch.equal(got.isnan(), want), (m, n, k)


def test_extreme_scales_multiply(api):
    """Scales 2^-127 and 2^127 of the operands: the product of values whose own scales are out of fp32's normal range."""
    m, n, k = 17, 33, 256
    rng = np.random.default_rng(9)
    data = [rng.integers(0, 256, api.mx_bytes(r, k), dtype=np.uint8) for r in (m, n)]
    for d, r, s in zip(data, (m, n), (0, 254)):
        d[api.mx_scales_offset(r, k):] = s
    a, b = (api.MxMatrix(torch.from_numpy(d).cuda(), r, k) for d, r in zip(data, (m, n)))
    want, bound = R.product(R.restored(data[0], m, k), R.restored(data[1], n, k))
    got = api.fh_mx_matmul(a, b, out_dtype=torch.float32).double().cpu().numpy()
    assert (np.abs(got - want) <= bound + R.U32 * np.abs(want)).all()


def test_the_three_products_of_a_layer_agree(api):
    """x by rows and by columns hold the same values only where their blocks agree; a matrix of one scale does, so the
    weight's gradient from the columns' forms equals the one from transposed copies."""
    rng = np.random.default_rng(4)
    x = torch.from_numpy(rng.choice(R.GRID[1:], (130, 70)).astype(np.float32)).cuda()
    g = torch.from_numpy(rng.choice(R.GRID[1:], (130, 50)).astype(np.float32)).cuda()
    x[::32], x[:, ::32], g[::32], g[:, ::32] = 6.0, 6.0, 6.0, 6.0
    _, xc = api.fh_mx_quantize(x, "both")
    _, gc = api.fh_mx_quantize(g, "both")
    got = api.fh_mx_matmul(gc, xc, out_dtype=torch.float32)
    assert torch.equal(got.cpu(), (g.double().t().cpu() @ x.double().cpu()).float())
    assert torch.equal(api.fh_mx_quantize(x.t().contiguous(), "rows").data[:70 * 128], xc.data[:70 * 128])


def test_calls_repeat_bit_for_bit(api):
    t, _ = _values(300, 700, 8)
    d = t.cuda()
    a = api.fh_mx_quantize(d, "both", "stochastic", 5, 6)
    b = api.fh_mx_quantize(d, "both", "stochastic", 5, 6)
    other = api.fh_mx_quantize(d, "rows", "stochastic", 5, 7)
    known = torch.from_numpy(R.stored(t.numpy())[1]).cuda()
    assert torch.equal(a[0].data[known], b[0].data[known]) and not torch.equal(a[0].data[known], other.data[known])
    x, w = api.fh_mx_quantize(d), api.fh_mx_quantize(d[:200])
    first = api.fh_mx_matmul(x, w)
    for _ in range(5):
        assert torch.equal(api.fh_mx_matmul(x, w), first)


def test_more_than_32_bits_of_elements(api):
    """Rows far beyond 2^31 elements and 2^32 bytes from the start come out as the same rows do alone."""
    print("[large] quantise", flush=True)
    rows, cols, tail = 70_001, 32_768, 40
    x = torch.zeros((rows, cols), dtype=torch.bfloat16, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(1)
    x[-tail:] = torch.randn((tail, cols), generator=g, device="cuda").bfloat16()
    m = api.fh_mx_quantize(x)
    alone = api.fh_mx_dequantize(api.fh_mx_quantize(x[-tail:]), torch.bfloat16)
    back = api.fh_mx_dequantize(m, torch.bfloat16)
    assert torch.equal(back[-tail:], alone)
    del back
    y, mean, rstd = api.fh_layer_norm(x)
    y2, mean2, rstd2 = api.fh_layer_norm(x[-tail:])
    assert torch.equal(y[-tail:], y2) and torch.equal(mean[-tail:], mean2) and torch.equal(rstd[-tail:], rstd2)
    del y
    print("[large] product", flush=True)
    w = api.fh_mx_quantize(torch.randn((40_000, 64), generator=g, device="cuda"))
    a = torch.randn((60_001, 64), generator=g, device="cuda")
    out = api.fh_mx_matmul(api.fh_mx_quantize(a), w)
    assert torch.equal(out[-tail:], api.fh_mx_matmul(api.fh_mx_quantize(a[-tail:]), w))


def test_on_a_side_stream(api):
    """Work enqueued on a stream that is not the current one, with allocations on the current one right behind it."""
    t, x = _values(512, 768, 3)
    d = t.cuda()
    qa = api.fh_mx_quantize(d, "columns")
    want = api.fh_mx_matmul(qa, qa, out_dtype=torch.float32)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for _ in range(3):
        q = api.fh_mx_quantize(d, "columns", stream=side)
        got = api.fh_mx_matmul(q, q, out_dtype=torch.float32, stream=side)
        for k in range(4):
            torch.empty(max(16, api.mx_matmul_workspace_bytes(768, 768, 512)), dtype=torch.uint8, device="cuda").fill_(k)
        side.synchronize()
        torch.cuda.synchronize()
        assert torch.equal(got, want)


def test_the_binding_refuses(api):
    x = torch.zeros(8, 64, device="cuda")
    m = api.fh_mx_quantize(x)
    with pytest.raises(TypeError):
        api.fh_mx_quantize(x.half())
    with pytest.raises(ValueError):
        api.fh_mx_quantize(x.t())
    with pytest.raises(ValueError):
        api.fh_mx_quantize(x[0])
    with pytest.raises(ValueError):
        api.fh_mx_quantize(x.expand(4, 8, 64)[:, 0].as_strided((4, 64), (0, 1)))
    with pytest.raises(KeyError):
        api.fh_mx_quantize(x, rounding="up")
    with pytest.raises(ValueError):
        api.fh_mx_matmul(m, api.fh_mx_quantize(x[:, :32]))
    with pytest.raises(ValueError):
        api.fh_mx_matmul(m, m, bias=torch.zeros(7, device="cuda"))
    with pytest.raises(ValueError):
        api.fh_mx_matmul(m, m, out=torch.zeros(8, 9, device="cuda"))
    with pytest.raises(ValueError):
        api.fh_mx_matmul(m, m, bias=torch.zeros(8))
    with pytest.raises(api.FedHybridError):
        api.fh_mx_dequantize(api.MxMatrix(m.data[:-1], 8, 64))
    with pytest.raises(ValueError):
        api.fh_mx_dequantize(m, out=torch.zeros(8, 63, device="cuda"))


@pytest.mark.parametrize("rows, cols", [(65536, 200), (65537, 200), (65539, 33), (32771, 300)])
def test_restored_values_of_many_rows(api, rows, cols):
    """Around the number of rows from which a lane takes several, the last ones fewer, into a view: exact products of codes and scales."""
    t, x = _values(rows, cols, rows)
    m = api.fh_mx_quantize(t.cuda())
    want = torch.from_numpy(R.restored(m.data.cpu().numpy(), rows, cols))
    for dtype in (torch.float32, torch.bfloat16):
        wide = torch.full((rows, cols + 3), 7.0, dtype=dtype, device="cuda")
        api.fh_mx_dequantize(m, out=wide[:, 1:1 + cols])
        assert torch.equal(wide[:, 1:1 + cols].cpu(), want.to(dtype)) and (wide[:, 0] == 7).all() and (wide[:, 1 + cols:] == 7).all()
