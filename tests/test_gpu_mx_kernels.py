"""Every kernel of the microscaled product against binary64 (computed on the GPU by torch from the restored operands), within the rounding of a
binary32 sum: R.product's bound, and half a step of the output's type."""
from __future__ import annotations

import numpy as np
import pytest

import mx_products as M
import mx_reference as R

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
IDS = ["-".join(str(v) for v in p if v is not None) for p in M.PRODUCTS]


@pytest.fixture(scope="module")
def api():
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a visible MI355X")
    from paper_2510_11400_amd import api as _api
    return _api


def _operand(api, rows, k, seed):
    """(a stored matrix of values on the grid, these values in binary64): codes of their own at scales 2^-6 .. 2^6, put into the stored form by the
    layout's definition alone."""
    rng = np.random.default_rng(seed)
    width = R.padded(k)
    data = rng.integers(0, 256, api.mx_bytes(rows, k), dtype=np.uint8)
    codes = data[:rows * width // 2].reshape(rows, width // 2)
    codes[:, (k + 1) // 2:] = 0
    if k % 2:
        codes[:, k // 2] &= 15
    scales = data[rows * width // 2:]
    at = R.scale_positions(rows, width)
    scales[:] = 255                                              # of rows past the last: never used
    scales[at] = rng.integers(121, 134, at.shape)
    packed = torch.from_numpy(codes).cuda()
    code = torch.stack((packed & 15, packed >> 4), -1).view(rows, width).long()
    grid = torch.tensor(list(R.GRID) + [-v for v in R.GRID], dtype=torch.float64, device="cuda")
    scale = torch.exp2(torch.from_numpy(scales[at].astype(np.float64)).cuda() - 127)
    return api.MxMatrix(torch.from_numpy(data).cuda(), rows, k), (grid[code] * scale.repeat_interleave(32, 1))[:, :k]


def _check(got, want, size, k, dtype, what):
    bound = (k / 32 + 32) * R.U32 * size
    far = (got.double() - want).abs()
    bad = (~(far <= bound + R.HALF_STEP[dtype] * (want.abs() + bound))).nonzero()
    assert bad.numel() == 0, f"{what}: {len(bad)} outputs off, first at {bad[0].tolist()}, last at {bad[-1].tolist()}"


@pytest.mark.parametrize("kernel, how, m, n, k", M.PRODUCTS, ids=IDS)
def test_products_of_every_kernel(api, kernel, how, m, n, k):
    """Both output types, without a bias and with one of either type, into a matrix of its own and into a view, whose neighbours stay."""
    print(f"[product] {kernel} {how} {m} {n} {k}", flush=True)
    (a, va), (b, vb) = _operand(api, m, k, m + k), _operand(api, n, k, n + k + 1)
    want, size = torch.mm(va, vb.t()), torch.mm(va.abs(), vb.abs().t())
    g = torch.Generator(device="cuda").manual_seed(m)
    for out, bias_dtype, view in (("bf16", "f32", False), ("f32", None, False), ("f32", "bf16", True), ("bf16", None, True)):
        bias = None if bias_dtype is None else (100 * torch.randn(n, generator=g, device="cuda")).to(DTYPES[bias_dtype])
        wide = torch.full((m, n + 9), 3.0, dtype=DTYPES[out], device="cuda") if view else None
        got = api.fh_mx_matmul(a, b, bias, DTYPES[out], out=wide[:, 5:5 + n] if view else None)
        full, most = (want, size) if bias is None else (want + bias.double(), size + bias.double().abs())
        _check(got, full, most, k, out, f"{kernel} {m} x {n} x {k}, {out}, bias {bias_dtype}, view {view}")
        if view:
            assert bool((wide[:, :5] == 3).all()) and bool((wide[:, 5 + n:] == 3).all())


@pytest.mark.parametrize("kernel, how, m, n, k", M.PRODUCTS, ids=IDS)
def test_broken_blocks_reach_their_rows_alone(api, kernel, how, m, n, k):
    """In every kernel: a block of NaN in the first, a middle and the last row of a and in a middle and the last row of b makes the sums of these rows NaN, the
    others are as they are without; and calls repeat bit for bit."""
    print(f"[broken] {kernel} {how} {m} {n} {k}", flush=True)
    (a, _), (b, _) = _operand(api, m, k, 1), _operand(api, n, k, 2)
    whole = api.fh_mx_matmul(a, b, out_dtype=torch.float32)
    for _ in range(3):
        again = api.fh_mx_matmul(a, b, out_dtype=torch.float32)
        assert torch.equal(again, whole)
    rows, cols = sorted({0, m // 2, m - 1}), sorted({n // 2, n - 1})
    blocks = (k + 31) // 32
    for q, broken in ((a, rows), (b, cols)):
        at = R.scale_positions(q.rows, R.padded(k))
        for i, r in enumerate(broken):
            q.data[api.mx_scales_offset(q.rows, k) + int(at[r, (i * 7919 + blocks // 2) % blocks])] = 255
    got = api.fh_mx_matmul(a, b, out_dtype=torch.float32)
    dead = torch.zeros((m, n), dtype=torch.bool, device="cuda")
    dead[rows], dead[:, cols] = True, True
    assert torch.equal(got.isnan(), dead)
    assert torch.equal(got.masked_fill(dead, 0.0), whole.masked_fill(dead, 0.0))
