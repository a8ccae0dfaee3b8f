"""The microscaled 4-bit operators and layer norm as measured cases.

A case is a dict of plain values; `prepare` makes the inputs on the GPU, `run` is one pass in plain torch operations
(`own` false) or through the public entry points (`own` true), `exact` the same result from the definition in binary64.
Kinds of case:

  quantise        fh_mx_quantize by rows, by columns or both, and fh_mx_dequantize of what was stored
  product         fh_mx_matmul of two stored matrices: a layer's forward product, its data or weight gradient
  norm            fh_layer_norm
  norm_backward   fh_layer_norm_backward: the input's gradient and the reductions of the weight's and the bias's
  serve           fh_layer_norm_mx + fh_mx_matmul on stored weights: a frozen layer answering a few tokens
  step            layers.layer_norm_mx_linear forward and backward: the training step of such a layer

A stored matrix of R rows and C columns (blocks of 32 values along a row, C padded to a multiple of 256) is one buffer:
R x C/2 bytes of codes (value c of a row in byte c/2, the even one in the low half), then a scale byte 2^(s-127) for each
block, in pieces of 32 rows x 8 blocks: byte ((r/32) * (C/256) + b/8) * 256 + (b%8 / 4) * 128 + (r%32) * 4 + b%4.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

_DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
_SIZE = {"f32": 4, "bf16": 2}
_EPS = 1e-5
_SEED, _TENSOR = 0x9E3779B97F4A7C15, 5


# ---- the cases ---------------------------------------------------------------------------------------
def listed():
    return [
        # the smallest call: a handful of tokens' activations of an encoder (hidden 768), saved and restored
        {"name": "quantise_tokens", "kind": "quantise", "rows": 17, "cols": 768, "dtype": "bf16", "form": "rows", "rounding": "nearest"},
        # a layer norm's output for a whole batch (16 x 512 tokens, hidden 768): a forward product's operand
        {"name": "quantise_encoder", "kind": "quantise", "rows": 8192, "cols": 768, "dtype": "bf16", "form": "rows", "rounding": "nearest"},
        # a gradient of odd size, kept for both backward products, stochastically rounded so that its mean survives
        {"name": "quantise_gradient", "kind": "quantise", "rows": 4095, "cols": 1000, "dtype": "f32", "form": "both", "rounding": "stochastic"},
        # one token through a frozen layer: the norm writes codes, the product reads them, weights are stored once
        {"name": "serve_token", "kind": "serve", "tokens": 1, "cols": 4096, "out": 4096, "bias": True},
        # a short prompt of ragged sizes
        {"name": "product_prompt", "kind": "product", "m": 197, "n": 1000, "k": 1537, "out": "f32", "bias": True},
        # the weight's gradient of an attention projection: few outputs, a sum over all 8192 tokens
        {"name": "product_weight_gradient", "kind": "product", "m": 768, "n": 768, "k": 8192, "out": "f32", "bias": False},
        # the largest: a wide layer's forward product over a long batch
        {"name": "product_large", "kind": "product", "m": 8192, "n": 8192, "k": 4096, "out": "bf16", "bias": True},
        # the encoder's layer norm, and a wide one of odd size in fp32
        {"name": "norm_encoder", "kind": "norm", "rows": 8192, "cols": 768, "dtype": "bf16", "params": "bf16"},
        {"name": "norm_wide", "kind": "norm", "rows": 1025, "cols": 12345, "dtype": "f32", "params": "f32"},
        # their backward passes
        {"name": "norm_backward_encoder", "kind": "norm_backward", "rows": 8192, "cols": 768, "dtype": "bf16", "params": "f32"},
        {"name": "norm_backward_wide", "kind": "norm_backward", "rows": 2047, "cols": 8193, "dtype": "f32", "params": "f32"},
        # all of it: the training step of a norm and the projection behind it (queries, keys and values: 3 x 768)
        {"name": "step_encoder", "kind": "step", "tokens": 8192, "cols": 768, "out": 2304},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(("quantise", "quantise", "product", "product", "product", "norm", "norm_backward", "norm_backward", "serve", "step"))
    case = {"kind": kind}
    if kind == "quantise":
        case["cols"] = _log(rng, 32, 8192)
        case["rows"] = min(_log(rng, 1, 16384), (1 << 23) // case["cols"])
        case.update(dtype=rng.choice(("f32", "bf16")), form=rng.choice(("rows", "columns", "both")),
                    rounding=rng.choice(("nearest", "stochastic")))
    elif kind == "product":
        case.update(m=_log(rng, 1, 8192), n=_log(rng, 16, 8192), k=_log(rng, 32, 8192), out=rng.choice(("f32", "bf16")),
                    bias=rng.random() < 0.5)
        case["k"] = min(case["k"], (1 << 38) // (case["m"] * case["n"]))
    elif kind in ("norm", "norm_backward"):
        case["cols"] = _log(rng, 32, 16384)
        case["rows"] = min(_log(rng, 1, 16384), (1 << 24) // case["cols"])
        case["dtype"] = rng.choice(("f32", "bf16"))
        case["params"] = rng.choice(("f32", case["dtype"]))
    elif kind == "serve":
        case.update(tokens=_log(rng, 1, 64), cols=_log(rng, 64, 8192), out=_log(rng, 64, 8192), bias=rng.random() < 0.5)
    else:
        case.update(tokens=_log(rng, 32, 8192), cols=_log(rng, 64, 2048), out=_log(rng, 64, 2560))
    return case


# ---- inputs --------------------------------------------------------------------------------------------
def _activation(g, rows, cols, dtype):
    """Values as layers meet them: every row with a mean and a width of its own, a few channels far wider than the rest."""
    x = torch.randn((rows, cols), generator=g, device="cuda")
    wide = (torch.rand(cols, generator=g, device="cuda") < 0.01).float() * 9.0 + 1.0
    row = torch.rand((rows, 1), generator=g, device="cuda")
    return ((x * (0.5 + row)) * wide + (row - 0.3)).to(dtype)


def _gradient(g, rows, cols, dtype):
    """A loss's gradient: small, and of another size in every row."""
    size = torch.exp(torch.randn((rows, 1), generator=g, device="cuda")) * 1e-3
    return (torch.randn((rows, cols), generator=g, device="cuda") * size).to(dtype)


def _parameters(g, cols, dtype):
    w = 1.0 + 0.2 * torch.randn(cols, generator=g, device="cuda")
    return w.to(dtype), (0.1 * torch.randn(cols, generator=g, device="cuda")).to(dtype)


def _weights(g, n, k):
    return torch.randn((n, k), generator=g, device="cuda") / math.sqrt(k)


def _padded(cols):
    return -(-cols // 256) * 256


def _stored(x):
    """The stored form of x, as a program holds a layer's weights or an operand that an earlier call left."""
    rows, cols = x.shape
    width = _padded(cols)
    s, q = _blocks(torch.nn.functional.pad(x.float(), (0, width - cols)))
    code = torch.searchsorted(torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0], device=x.device), q.abs())
    code = (code + torch.where(q < 0, 8, 0)).to(torch.uint8).view(rows, width // 2, 2)
    scales = torch.nn.functional.pad((s + 127).to(torch.uint8).view(rows, width // 32), (0, 0, 0, -rows % 32))
    scales = scales.view(-1, 32, width // 256, 2, 4).permute(0, 2, 3, 1, 4).reshape(-1)
    return torch.cat(((code[..., 0] | code[..., 1] << 4).reshape(-1), scales))


def prepare(case, seed):
    kind = case["kind"]
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    state = {"case": case}
    if kind == "quantise":
        make = _gradient if case["rounding"] == "stochastic" else _activation
        state["x"] = make(g, case["rows"], case["cols"], _DTYPES[case["dtype"]])
    elif kind == "product":
        state["a"] = _stored(_activation(g, case["m"], case["k"], torch.float32))
        state["b"] = _stored(_weights(g, case["n"], case["k"]))
        state["bias"] = torch.randn(case["n"], generator=g, device="cuda") if case["bias"] else None
    elif kind in ("norm", "norm_backward"):
        state["x"] = _activation(g, case["rows"], case["cols"], _DTYPES[case["dtype"]])
        state["weight"], state["bias"] = _parameters(g, case["cols"], _DTYPES[case["params"]])
        if kind == "norm_backward":
            state["dy"] = _gradient(g, case["rows"], case["cols"], _DTYPES[case["dtype"]])
            x = state["x"].double()                          # what the forward pass left
            state["mean"] = x.mean(1).float()
            state["rstd"] = torch.rsqrt(x.var(1, unbiased=False) + _EPS).float()
    elif kind == "serve":
        state["x"] = _activation(g, case["tokens"], case["cols"], torch.bfloat16)
        state["weight"], state["bias"] = _parameters(g, case["cols"], torch.bfloat16)
        state["w"] = _stored(_weights(g, case["out"], case["cols"]))
        state["out_bias"] = torch.randn(case["out"], generator=g, device="cuda").bfloat16() if case["bias"] else None
    else:
        state["x"] = _activation(g, case["tokens"], case["cols"], torch.bfloat16).requires_grad_()
        state["weight"], state["bias"] = (p.requires_grad_() for p in _parameters(g, case["cols"], torch.bfloat16))
        state["w"] = _weights(g, case["out"], case["cols"]).bfloat16().requires_grad_()
        state["dy"] = _gradient(g, case["tokens"], case["out"], torch.bfloat16)
    return state


# ---- the plain forms: torch operations in 32 bits --------------------------------------------------------
def _blocks(x, u=None):
    """(exponents, quantised values over their scale) of the blocks of 32 along the rows; u: 16 random bits a value."""
    v = x.view(x.shape[0], -1, 32)
    top = v.abs().amax(-1, keepdim=True)
    s = (torch.frexp(top)[1] - 3).clamp(min=-126)
    s = torch.where(top == 0, -126, s)
    t = torch.ldexp(v.abs(), -s).clamp(max=6.0)
    step = torch.where(t < 2, 0.5, torch.where(t < 4, 1.0, 2.0))
    if u is None:
        q = torch.round(t / step) * step
    else:
        low = torch.floor(t / step)
        part = torch.round((t / step - low) * 2.0 ** 22)
        q = (low + (part > 64.0 * u.view(v.shape)).float()) * step
    return s, torch.copysign(q, v)


def _quantised(x, u=None):
    """x in 32 bits, rounded to blocks along its rows."""
    rows, cols = x.shape
    pad = (0, -cols % 32)
    s, q = _blocks(torch.nn.functional.pad(x, pad), None if u is None else torch.nn.functional.pad(u, pad))
    return torch.ldexp(q, s).view(rows, -1)[:, :cols]


def _random_bits(rows, cols, device):
    """16 random bits a value: Philox4x32-10, a block of eight half-words for eight rows of a column."""
    low = 0xFFFFFFFF
    at = torch.arange(-(-rows // 8) * cols, device=device, dtype=torch.int64)
    c0, c1, c2, c3 = at & low, at >> 32, torch.full_like(at, _TENSOR & low), torch.full_like(at, _TENSOR >> 32)
    k0, k1 = _SEED & low, _SEED >> 32
    for _ in range(10):
        p0, p1 = c0 * 0xD2511F53, c2 * 0xCD9E8D57
        c0, c1, c2, c3 = ((p1 >> 32) & low) ^ c1 ^ k0, p1 & low, ((p0 >> 32) & low) ^ c3 ^ k1, p0 & low
        k0, k1 = (k0 + 0x9E3779B9) & low, (k1 + 0xBB67AE85) & low
    halves = torch.stack((c0 & 0xFFFF, c0 >> 16, c1 & 0xFFFF, c1 >> 16, c2 & 0xFFFF, c2 >> 16, c3 & 0xFFFF, c3 >> 16))
    return halves.view(8, -1, cols).transpose(0, 1).reshape(-1, cols)[:rows].float()


def _values(buffer, rows, cols):
    """The values that a stored matrix stands for, in 32 bits."""
    width = _padded(cols)
    codes = buffer[:rows * width // 2].view(rows, width // 2)
    scales = buffer[rows * width // 2:].view(-1, width // 256, 2, 32, 4).permute(0, 3, 1, 2, 4).reshape(-1, width // 32)[:rows]
    grid = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], device=buffer.device)
    grid = torch.cat((grid, -grid))
    v = grid[torch.stack((codes & 15, codes >> 4), -1).view(rows, width).int()]
    scale = torch.ldexp(torch.ones_like(scales, dtype=torch.float32), scales.int() - 127)
    return (v.view(rows, -1, 32) * scale[..., None]).view(rows, width)[:, :cols]


def _norm(x, weight, bias):
    x = x.float()
    mean = x.mean(1, keepdim=True)
    rstd = torch.rsqrt((x - mean).square().mean(1, keepdim=True) + _EPS)
    return (x - mean) * rstd * weight.float() + bias.float(), mean, rstd


def _norm_backward(dy, x, mean, rstd, weight):
    h = (x.float() - mean) * rstd
    g = dy * weight.float()
    dx = rstd * (g - g.mean(1, keepdim=True) - h * (g * h).mean(1, keepdim=True))
    return dx, (dy * h).sum(0), dy.sum(0)


def _run_plain(state):
    case, kind = state["case"], state["case"]["kind"]
    if kind == "quantise":
        x = state["x"].float()
        u = _random_bits(*x.shape, x.device) if case["rounding"] == "stochastic" else None
        out = []
        if case["form"] in ("rows", "both"):
            out.append(_quantised(x, u).to(state["x"].dtype))
        if case["form"] in ("columns", "both"):
            out.append(_quantised(x.t().contiguous(), None if u is None else u.t().contiguous()).to(state["x"].dtype))
        return out
    if kind == "product":
        y = _values(state["a"], case["m"], case["k"]) @ _values(state["b"], case["n"], case["k"]).t()
        return (y if state["bias"] is None else y + state["bias"]).to(_DTYPES[case["out"]])
    if kind == "norm":
        y, mean, rstd = _norm(state["x"], state["weight"], state["bias"])
        return y.to(state["x"].dtype), mean.view(-1), rstd.view(-1)
    if kind == "norm_backward":
        dx, dw, db = _norm_backward(state["dy"].float(), state["x"], state["mean"][:, None], state["rstd"][:, None], state["weight"])
        return dx.to(state["x"].dtype), dw.to(state["weight"].dtype), db.to(state["weight"].dtype)
    if kind == "serve":
        h = _quantised(_norm(state["x"], state["weight"], state["bias"])[0])
        y = h @ _values(state["w"], case["out"], case["cols"]).t()
        return (y if state["out_bias"] is None else y + state["out_bias"].float()).bfloat16()
    with torch.no_grad():
        x, weight, bias, w, dy = state["x"], state["weight"], state["bias"], state["w"].float(), state["dy"].float()
        h, mean, rstd = _norm(x, weight, bias)
        y = _quantised(h) @ _quantised(w).t()
        dh = _quantised(dy) @ _quantised(w.t().contiguous()).t()
        dw = _quantised(dy.t().contiguous()) @ _quantised(h.t().contiguous()).t()
        dx, dweight, dbias = _norm_backward(dh, x, mean, rstd, weight)
        return [v.bfloat16() for v in (y, dx, dweight, dbias, dw)]


# ---- the framework's calls -------------------------------------------------------------------------------
def _run_own(state):
    from paper_2510_11400_amd import api, layers
    case, kind = state["case"], state["case"]["kind"]
    if kind == "quantise":
        x = state["x"]
        kept = api.fh_mx_quantize(x, forms=case["form"], rounding=case["rounding"], seed=_SEED, tensor_id=_TENSOR)
        return [api.fh_mx_dequantize(m, out_dtype=x.dtype) for m in (kept if case["form"] == "both" else (kept,))]
    if kind == "product":
        a = api.MxMatrix(state["a"], case["m"], case["k"])
        b = api.MxMatrix(state["b"], case["n"], case["k"])
        return api.fh_mx_matmul(a, b, bias=state["bias"], out_dtype=_DTYPES[case["out"]])
    if kind == "norm":
        return api.fh_layer_norm(state["x"], state["weight"], state["bias"], eps=_EPS)
    if kind == "norm_backward":
        return api.fh_layer_norm_backward(state["dy"], state["x"], state["mean"], state["rstd"], state["weight"])
    if kind == "serve":
        h, _, _ = api.fh_layer_norm_mx(state["x"], state["weight"], state["bias"], eps=_EPS, forms="rows")
        w = api.MxMatrix(state["w"], case["out"], case["cols"])
        return api.fh_mx_matmul(h, w, bias=state["out_bias"], out_dtype=torch.bfloat16)
    leaves = (state["x"], state["weight"], state["bias"], state["w"])
    y = layers.layer_norm_mx_linear(*leaves, eps=_EPS)
    return [y.detach(), *torch.autograd.grad(y, leaves, state["dy"])]


def run(state):
    return _run_own(state) if own else _run_plain(state)


# ---- what a pass cannot do without ---------------------------------------------------------------------
def _mx_bytes(rows, cols):
    return rows * cols // 2 + rows * -(-cols // 32)


def work(case):
    """Every input read once, every output written once; what is stored in between is written and read back."""
    kind = case["kind"]
    if kind == "quantise":
        n, forms = case["rows"] * case["cols"], 2 if case["form"] == "both" else 1
        stored = _mx_bytes(case["rows"], case["cols"])
        return {"bytes": n * _SIZE[case["dtype"]] * (1 + forms) + 2 * forms * stored, "flops": 8 * n * forms}
    if kind == "product":
        m, n, k = case["m"], case["n"], case["k"]
        return {"bytes": _mx_bytes(m, k) + _mx_bytes(n, k) + m * n * _SIZE[case["out"]], "flops": 2 * m * n * k}
    if kind in ("norm", "norm_backward"):
        n, size, backward = case["rows"] * case["cols"], _SIZE[case["dtype"]], kind == "norm_backward"
        return {"bytes": n * size * (3 if backward else 2) + 8 * case["rows"] + (3 if backward else 2) * case["cols"] * _SIZE[case["params"]],
                "flops": n * (16 if backward else 8)}
    t, c, o = case["tokens"], case["cols"], case["out"]
    if kind == "serve":
        return {"bytes": 2 * t * c + _mx_bytes(t, c) + _mx_bytes(o, c) + 2 * t * o, "flops": 2 * t * c * o + 16 * t * c}
    # x, dy, dx, y, w and its gradient once; both forms of the norm's output, of dy and of w written and read; dh written and read
    stored = 4 * (_mx_bytes(t, c) + _mx_bytes(t, o) + _mx_bytes(o, c))
    return {"bytes": 2 * (2 * t * c + 2 * t * o + 2 * o * c) + stored + 4 * t * c, "flops": 6 * t * c * o + 40 * t * c}


# ---- the same in binary64 ------------------------------------------------------------------------------
_GRID = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _rounded64(x, u=None):
    """x (binary64) with every run of 32 values of a row on the grid of its scale; u: random numbers in [0, 1)."""
    rows, cols = x.shape
    out = torch.empty_like(x)
    whole = cols // 32 * 32
    for lo, hi, width in ((0, whole, 32), (whole, cols, cols - whole)):
        if lo == hi or not rows:
            continue
        v = x[:, lo:hi].reshape(-1, width)
        top = v.abs().max(1, keepdim=True).values
        scale = torch.exp2((torch.floor(torch.log2(top.clamp(min=2.0 ** -149))) - 2).clamp(min=-126))
        t = v.abs() / scale
        near = torch.zeros_like(t)
        for k in range(7):
            a, b = _GRID[k], _GRID[k + 1]
            if u is None:
                up = (t > (a + b) / 2) | ((t == (a + b) / 2) & (k % 2 == 1))
            else:                                                # the fraction counts in steps of 2^-22
                up = torch.round((t - a) / (b - a) * 2 ** 22) > u[:, lo:hi].reshape(-1, width) * 2 ** 22
            near = torch.where((t >= a) & up, b, torch.where(t >= a, a, near))
        near = torch.where(t >= 6, 6.0, near)
        out[:, lo:hi] = (torch.sign(v) * near * scale).view(rows, hi - lo)
    return out


def _uniform64(rows, cols):
    """The random number of every value, by Philox4x32-10 on the host."""
    n = -(-rows // 8) * cols
    word = [np.arange(n, dtype=np.uint64) & np.uint64(0xFFFFFFFF), np.arange(n, dtype=np.uint64) >> np.uint64(32),
            np.full(n, _TENSOR & 0xFFFFFFFF, np.uint64), np.full(n, _TENSOR >> 32, np.uint64)]
    key = [_SEED & 0xFFFFFFFF, _SEED >> 32]
    low, half = np.uint64(0xFFFFFFFF), np.uint64(32)
    for _ in range(10):
        a, b = word[0] * np.uint64(0xD2511F53), word[2] * np.uint64(0xCD9E8D57)
        word = [(b >> half) ^ word[1] ^ np.uint64(key[0]), b & low, (a >> half) ^ word[3] ^ np.uint64(key[1]), a & low]
        key = [(key[0] + 0x9E3779B9) & 0xFFFFFFFF, (key[1] + 0xBB67AE85) & 0xFFFFFFFF]
    bits = np.stack(word, 1).astype(np.uint32).view(np.uint16).reshape(-1, cols, 8)      # [eight rows][column][half-word]
    u = bits.transpose(0, 2, 1).reshape(-1, cols)[:rows].astype(np.float64) / 65536.0
    return torch.from_numpy(u).cuda()


def _decoded64(buffer, rows, cols):
    width = _padded(cols)
    codes = buffer[:rows * width // 2].view(rows, -1).int()
    n = torch.empty((rows, width), dtype=torch.int32, device=buffer.device)
    n[:, 0::2], n[:, 1::2] = codes % 16, codes // 16
    e, m = n // 2 % 4, (n % 2).double()
    v = torch.where(e == 0, m / 2, (1 + m / 2) * torch.exp2(e.double() - 1)) * (1.0 - 2.0 * (n // 8))
    r = torch.arange(rows, device=buffer.device)[:, None]
    b = torch.arange(width // 32, device=buffer.device)[None]
    at = (r // 32 * (width // 256) + b // 8) * 256 + b % 8 // 4 * 128 + r % 32 * 4 + b % 4
    scale = torch.exp2(buffer[rows * width // 2:][at].double() - 127)
    return (v * scale.repeat_interleave(32, 1))[:, :cols]


def _norm64(x, weight, bias):
    x = x.double()
    mean = x.sum(1, keepdim=True) / x.shape[1]
    rstd = 1.0 / torch.sqrt(((x - mean) ** 2).sum(1, keepdim=True) / x.shape[1] + _EPS)
    return (x - mean) * rstd * weight.double() + bias.double(), mean, rstd


def _norm_backward64(dy, x, mean, rstd, weight):
    n = x.shape[1]
    h, g = (x.double() - mean) * rstd, dy * weight.double()
    dx = rstd / n * (n * g - g.sum(1, keepdim=True) - h * (g * h).sum(1, keepdim=True))
    return dx, (dy * h).sum(0), dy.sum(0)


def exact(case, seed):
    kind, state = case["kind"], prepare(case, seed)
    with torch.no_grad():
        if kind == "quantise":
            x = state["x"].double()
            u = _uniform64(*x.shape) if case["rounding"] == "stochastic" else None
            out = []
            if case["form"] != "columns":
                out.append(_rounded64(x, u))
            if case["form"] != "rows":
                out.append(_rounded64(x.t().contiguous(), None if u is None else u.t().contiguous()))
            return out
        if kind == "product":
            y = torch.mm(_decoded64(state["a"], case["m"], case["k"]), _decoded64(state["b"], case["n"], case["k"]).t())
            return y if state["bias"] is None else y + state["bias"].double()
        if kind == "norm":
            y, mean, rstd = _norm64(state["x"], state["weight"], state["bias"])
            return y, mean.view(-1), rstd.view(-1)
        if kind == "norm_backward":
            return _norm_backward64(state["dy"].double(), state["x"], state["mean"].double()[:, None], state["rstd"].double()[:, None],
                                    state["weight"])
        if kind == "serve":
            h = _rounded64(_norm64(state["x"], state["weight"], state["bias"])[0])
            y = torch.mm(h, _decoded64(state["w"], case["out"], case["cols"]).t())
            return y if state["out_bias"] is None else y + state["out_bias"].double()
        w, dy = state["w"].double(), state["dy"].double()
        h, mean, rstd = _norm64(state["x"], state["weight"], state["bias"])
        y = torch.mm(_rounded64(h), _rounded64(w).t())
        dh = torch.mm(_rounded64(dy), _rounded64(w.t().contiguous()).t())
        dw = torch.mm(_rounded64(dy.t().contiguous()), _rounded64(h.t().contiguous()).t())
        dx, dweight, dbias = _norm_backward64(dh, state["x"], mean, rstd, state["weight"])
        return [y, dx, dweight, dbias, dw]
