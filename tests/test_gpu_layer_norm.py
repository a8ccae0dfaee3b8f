"""Layer norm and its backward pass on the GPU against binary64, within the rounding of binary32 sums (bounds derived in
mx_reference), and with codes in place of its output against the dense output quantised."""
from __future__ import annotations

import numpy as np
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


def _inputs(rows, cols, dtype, p_dtype, seed):
    rng = np.random.default_rng(seed)
    x = rng.standard_normal((rows, cols)) * np.exp2(rng.integers(-6, 6, (rows, 1))) + rng.standard_normal((rows, 1)) * 3
    dy = rng.standard_normal((rows, cols)) * np.exp2(rng.integers(-10, 4, (rows, 1)))
    t, g = (torch.from_numpy(v.astype(np.float32)).to(DTYPES[dtype]) for v in (x, dy))
    w, b = (torch.from_numpy(v.astype(np.float32)).to(DTYPES[p_dtype]) for v in (1 + 0.3 * rng.standard_normal(cols), rng.standard_normal(cols)))
    return t, g, w, b


def _within(got, want, bound, dtype, what):
    far = np.abs(got.double().cpu().numpy() - want)
    bound = bound + R.HALF_STEP[dtype] * (np.abs(want) + bound) + 1e-38
    bad = np.argwhere(~(far <= bound))
    assert bad.size == 0, f"{what}: {len(bad)} of {want.size} off, first at {bad[0]}: {far[tuple(bad[0])]:.3g} over {bound[tuple(bad[0])]:.3g}"


def _check_forward(api, t, w, b, eps, dtype, out=None):
    x = t.double().numpy()
    weight, bias = (np.full(x.shape[1], v) if p is None else p.double().numpy() for p, v in ((w, 1.0), (b, 0.0)))
    y, mean, rstd, d_y, d_mean, d_rstd = R.layer_norm(x, weight, bias, float(np.float32(eps)))
    cuda = lambda v: None if v is None else v.cuda()  # noqa: E731
    got = api.fh_layer_norm(t.cuda(), cuda(w), cuda(b), eps, out=out)
    _within(got[0], y, d_y, dtype, f"y of {x.shape}")
    _within(got[1], mean, d_mean, "f32", f"mean of {x.shape}")
    _within(got[2], rstd, d_rstd, "f32", f"rstd of {x.shape}")
    return got


SHAPES = [(1, 1), (3, 2), (1, 7), (5, 8), (4, 63), (9, 64), (1, 511), (6, 512), (7, 513), (3, 768), (1030, 40), (2, 1024), (5, 1025),
          (3, 2048), (2, 2049), (3, 4096), (2, 4097), (3, 8192), (1, 8200), (2, 12345), (1, 16384), (2, 16385), (1, 30001)]


@pytest.mark.parametrize("params", ["f32", "bf16"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_forward(api, dtype, params):
    for i, (rows, cols) in enumerate(SHAPES):
        t, _, w, b = _inputs(rows, cols, dtype, params, i)
        _check_forward(api, t, w, b, 1e-5, dtype)


@pytest.mark.parametrize("cols", [40, 777, 3000, 20000])
def test_forward_without_parameters(api, cols):
    t, _, w, b = _inputs(5, cols, "f32", "f32", 1)
    _check_forward(api, t, None, None, 1e-5, "f32")
    _check_forward(api, t, w, None, 1e-3, "f32")
    _check_forward(api, t, None, b, 0.0, "f32")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_forward_into_and_from_views(api, dtype):
    for cols, at in ((100, 1), (999, 3), (5000, 7)):
        t, _, w, b = _inputs(9, cols + 10, dtype, "f32", cols)
        x = t.cuda()[:, at:at + cols]
        wide = torch.full((9, cols + 6), 2.0, dtype=DTYPES[dtype], device="cuda")
        y, mean, _ = api.fh_layer_norm(x, w[:cols].cuda(), b[:cols].cuda(), out=wide[:, 5:5 + cols])
        alone, mean2, _ = _check_forward(api, t[:, at:at + cols].contiguous(), w[:cols], b[:cols], 1e-5, dtype)
        assert torch.equal(y, alone) and torch.equal(mean, mean2)
        assert (wide[:, :5] == 2).all() and (wide[:, 5 + cols:] == 2).all()
        same = x.contiguous()
        api.fh_layer_norm(same, w[:cols].cuda(), b[:cols].cuda(), out=same)
        assert torch.equal(same, alone)


def test_forward_of_a_mean_far_from_zero(api):
    """Values of 4096 +- 1: the variance is taken of what is left of the mean, and keeps its digits."""
    rng = np.random.default_rng(1)
    for cols in (768, 3000, 20000):
        t = torch.from_numpy((4096 + rng.standard_normal((4, cols))).astype(np.float32))
        _, _, rstd = api.fh_layer_norm(t.cuda())
        want = 1.0 / np.sqrt(t.double().numpy().var(1) + 1e-5)
        # the mean is off by 65 half steps of 4096 at most, which the variance takes squared: 65 * 2^-24 * 4096 = 0.016
        assert (np.abs(rstd.cpu().numpy() / want - 1) < 0.5 * (0.016 ** 2 + 2 * 2.0 ** -12) + 1e-5).all()


def test_constant_rows_and_broken_values(api):
    x = torch.ones(6, 300, device="cuda") * 3
    x[1, 5], x[2, 7], x[3, 9] = float("nan"), float("inf"), float("-inf")
    y, mean, rstd = api.fh_layer_norm(x, eps=1e-5)
    assert not y[0].any() and not y[4:].any() and mean[0] == 3
    assert torch.allclose(rstd[[0, 4, 5]], torch.full((3,), 1e-5 ** -0.5, device="cuda"), rtol=1e-6)
    assert y[1:4].isnan().all() and rstd[1:4].isnan().all()
    q, _, _ = api.fh_layer_norm_mx(x, forms="both")
    back = api.fh_mx_dequantize(q[0])
    assert back[1:4].isnan().all() and not back[0].any() and not back[4:].any()
    assert api.fh_mx_dequantize(q[1]).isnan().all()                       # every column's block holds one of those rows


def test_no_rows(api):
    x = torch.empty(0, 70, device="cuda")
    y, mean, rstd = api.fh_layer_norm(x)
    assert y.shape == (0, 70) and mean.shape == rstd.shape == (0,)
    dx, dw, db = api.fh_layer_norm_backward(x, x, mean, rstd, torch.ones(70, device="cuda"))
    assert dx.shape == (0, 70) and dw.shape == (70,) and not dw.any() and not db.any()


def _check_backward(api, t, g, w, dtype, p_dtype, seed, sums=True, **more):
    x, dy = t.double().numpy(), g.double().numpy()
    mean = torch.from_numpy(x.mean(1)).float()
    rstd = torch.from_numpy(1.0 / np.sqrt(x.var(1) + 1e-5)).float()
    weight = np.ones(x.shape[1]) if w is None else w.double().numpy()
    want = R.layer_norm_backward(dy, x, mean.double().numpy(), rstd.double().numpy(), weight)
    got = api.fh_layer_norm_backward(g.cuda(), t.cuda(), mean.cuda(), rstd.cuda(), None if w is None else w.cuda(), sums=sums, **more)
    _within(got[0], want[0], want[3], dtype, f"dx of {x.shape}")
    if sums:
        _within(got[1], want[1], want[4], p_dtype, f"dweight of {x.shape}")
        _within(got[2], want[2], want[5], p_dtype, f"dbias of {x.shape}")
    else:
        assert got[1] is None and got[2] is None
    return got


BACKWARD = SHAPES + [(5000, 33), (1025, 768), (300, 2000), (700, 3000), (600, 5000), (300, 9000), (270, 17000)]


@pytest.mark.parametrize("params", ["f32", "bf16"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_backward(api, dtype, params):
    for i, (rows, cols) in enumerate(BACKWARD):
        t, g, w, _ = _inputs(rows, cols, dtype, params, i)
        _check_backward(api, t, g, w, dtype, params, i)


@pytest.mark.parametrize("rows, cols", [(70, 100), (300, 3000), (20, 20000)])
def test_backward_of_part_of_it(api, rows, cols):
    t, g, w, _ = _inputs(rows, cols, "f32", "f32", 3)
    whole = _check_backward(api, t, g, None, "f32", "f32", 3)
    part = _check_backward(api, t, g, None, "f32", "f32", 3, sums=False)
    assert torch.equal(whole[0], part[0])
    for _ in range(3):
        again = _check_backward(api, t, g, None, "f32", "f32", 3)
        assert all(torch.equal(a, b) for a, b in zip(whole, again))


@pytest.mark.parametrize("rows, cols", [(70, 100), (300, 3000), (20, 20000)])
def test_backward_in_place_of_the_gradient(api, rows, cols):
    """dx in dy's own memory: the sums of dy are taken all the same."""
    t, g, w, _ = _inputs(rows, cols, "bf16", "f32", 4)
    apart = _check_backward(api, t, g, w, "bf16", "f32", 4)
    x = t.double().numpy()
    mean, rstd = torch.from_numpy(x.mean(1)).float().cuda(), torch.from_numpy(1.0 / np.sqrt(x.var(1) + 1e-5)).float().cuda()
    dy = g.cuda()
    got = api.fh_layer_norm_backward(dy, t.cuda(), mean, rstd, w.cuda(), dx=dy)
    assert got[0].data_ptr() == dy.data_ptr() and all(torch.equal(a, b) for a, b in zip(apart, got))


def test_backward_of_views(api):
    rows, cols = 40, 333
    t, g, w, _ = _inputs(rows, cols + 8, "bf16", "f32", 6)
    a = _check_backward(api, t[:, 3:3 + cols].contiguous(), g[:, 5:5 + cols].contiguous(), w[:cols], "bf16", "f32", 6)
    x = t[:, 3:3 + cols].double().numpy()
    mean, rstd = torch.from_numpy(x.mean(1)).float().cuda(), torch.from_numpy(1.0 / np.sqrt(x.var(1) + 1e-5)).float().cuda()
    wide = torch.full((rows, cols + 4), 7.0, dtype=torch.bfloat16, device="cuda")
    b = api.fh_layer_norm_backward(g.cuda()[:, 5:5 + cols], t.cuda()[:, 3:3 + cols], mean, rstd, w[:cols].cuda(), dx=wide[:, 1:1 + cols])
    assert all(torch.equal(p, q) for p, q in zip(a, b))
    assert (wide[:, 0] == 7).all() and (wide[:, 1 + cols:] == 7).all()


def test_backward_against_differences(api):
    """sum(dy * y) of the norm in binary64, moved by +- 1e-4 in one input at a time: the third derivative's share of such a
    difference is below 1e-8 of the gradient's size here, its rounding below 1e-10."""
    rng = np.random.default_rng(8)
    rows, cols, step = 4, 48, 1e-4
    x, dy, w = (rng.standard_normal(s).astype(np.float32) for s in ((rows, cols), (rows, cols), (cols,)))
    xd, gd, wd = (torch.from_numpy(v).cuda() for v in (x, dy, w))
    _, mean, rstd = api.fh_layer_norm(xd, wd, None, 1e-5)
    dx, dw, db = api.fh_layer_norm_backward(gd, xd, mean, rstd, wd)

    def loss(x, w, b):
        d = x - x.mean(1, keepdims=True)
        return float((dy.astype(float) * (d / np.sqrt((d * d).mean(1, keepdims=True) + 1e-5) * w + b)).sum())

    x, w, b = x.astype(float), w.astype(float), np.zeros(cols)

    def slope(v, at):
        up, down = v.copy(), v.copy()
        up[at], down[at] = v[at] + step, v[at] - step
        args = lambda u: (u if v is x else x, u if v is w else w, u if v is b else b)  # noqa: E731
        return (loss(*args(up)) - loss(*args(down))) / (2 * step)

    bounds = R.layer_norm_backward(dy.astype(float), x, mean.double().cpu().numpy(), rstd.double().cpu().numpy(), w)
    # the statistics are the kernel's own: off by a few half steps, which moves dx in proportion
    for at in [(i, j) for i in range(rows) for j in range(0, cols, 5)]:
        assert abs(float(dx[at]) - slope(x, at)) < bounds[3][at] + 1e-5 * np.abs(bounds[0]).max()
    for j in range(cols):
        assert abs(float(dw[j]) - slope(w, j)) < bounds[4][j] + 1e-5 * np.abs(bounds[1]).max()
        assert abs(float(db[j]) - slope(b, j)) < bounds[5][j] + 1e-5 * np.abs(bounds[2]).max()


@pytest.mark.parametrize("rounding", ["nearest", "stochastic"])
@pytest.mark.parametrize("forms", ["rows", "columns", "both"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_codes_are_those_of_the_output(api, dtype, forms, rounding):
    """The stored form is fh_mx_quantize's of the norm's binary32 output; for a bf16 input that is the output of the same
    values in fp32."""
    for i, (rows, cols) in enumerate([(1, 768), (3, 40), (33, 300), (260, 1000), (70, 2100), (40, 4100), (3, 9000), (2, 17000), (300, 64)]):
        t, _, w, b = _inputs(rows, cols, dtype, "f32", i)
        y, mean, rstd = api.fh_layer_norm(t.float().cuda(), w.cuda(), b.cuda())
        want = api.fh_mx_quantize(y, forms, rounding, 77, 5)
        got, mean2, rstd2 = api.fh_layer_norm_mx(t.cuda(), w.cuda(), b.cuda(), forms=forms, rounding=rounding, seed=77, tensor_id=5)
        assert torch.equal(mean, mean2) and torch.equal(rstd, rstd2)
        for a, c in zip(*((v if forms == "both" else (v,)) for v in (want, got))):
            known = torch.from_numpy(R.stored(np.zeros((a.rows, a.cols), np.float32))[1]).cuda()
            assert torch.equal(a.data[known], c.data[known]), (rows, cols)


def test_codes_without_parameters_from_views(api):
    t, _, _, _ = _inputs(50, 300, "bf16", "f32", 1)
    x = t.cuda()[:, 3:3 + 270]
    y, _, _ = api.fh_layer_norm(x.float())
    for forms in ("rows", "columns"):
        got, _, _ = api.fh_layer_norm_mx(x, forms=forms)
        assert torch.equal(api.fh_mx_dequantize(got), api.fh_mx_dequantize(api.fh_mx_quantize(y, forms)))


@pytest.mark.parametrize("params", ["f32", "bf16"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_codes_by_columns_of_every_width(api, dtype, params):
    """Around every limit on the columns and the rows, from rows that are not next to each other: both forms are those of the fp32
    output's, whichever kernels made them, and the form by rows is the one that is made alone."""
    for i, (rows, cols) in enumerate([(1, 1), (31, 255), (32, 256), (33, 257), (64, 512), (65, 513), (257, 767), (520, 1023), (290, 1024), (40, 1025), (300, 1536),
                                      (96, 1537), (513, 2047), (255, 2048), (34, 2049)]):
        t, _, w, b = _inputs(rows, cols + 5, dtype, params, i)
        x, w, b = t.cuda()[:, 2:2 + cols], w[:cols].cuda(), b[:cols].cuda()
        y, mean, rstd = api.fh_layer_norm(x.float(), w, b)
        (r, c), mean2, rstd2 = api.fh_layer_norm_mx(x, w, b, forms="both")
        alone = api.fh_layer_norm_mx(x, w, b, forms="columns")[0], api.fh_layer_norm_mx(x, w, b, forms="rows")[0]
        assert torch.equal(mean, mean2) and torch.equal(rstd, rstd2), (rows, cols)
        for m, want in zip((r, c, *alone), (*api.fh_mx_quantize(y, "both"), api.fh_mx_quantize(y, "columns"), api.fh_mx_quantize(y, "rows"))):
            known = torch.from_numpy(R.stored(np.zeros((m.rows, m.cols), np.float32))[1]).cuda()
            assert torch.equal(m.data[known], want.data[known]), (rows, cols)


def test_codes_of_broken_rows(api):
    """A row with a NaN or an infinity is NaN everywhere, and so is the block of every column that it is in, and nothing else."""
    x = torch.randn(100, 300, device="cuda")
    x[40, 7], x[97, 299] = float("nan"), float("inf")
    (r, c), _, _ = api.fh_layer_norm_mx(x, forms="both")
    by_rows, by_columns = torch.isnan(api.fh_mx_dequantize(r)), torch.isnan(api.fh_mx_dequantize(c))
    assert by_rows[[40, 97]].all() and int(by_rows.sum()) == 600
    assert by_columns[:, 32:64].all() and by_columns[:, 96:].all() and int(by_columns.sum()) == 300 * 36
