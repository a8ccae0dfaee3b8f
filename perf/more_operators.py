"""Storage in 8-bit integers, its product and the gated projection as measured cases.

A case is a dict of plain values; `prepare` makes the inputs on the GPU, `run` is one pass in plain torch operations
(`own` false) or through the public entry points (`own` true), `exact` the same result from the definition in binary64.
Kinds of case:

  quantise   fh_q8_quantize, and fh_q8_dequantize of what was stored
  product    fh_q8_matmul of two stored matrices: a served layer's product
  serve      fh_q8_quantize + fh_q8_gated on stored weights: a frozen gated layer answering tokens
  gated      fh_gated: act(x Wg^T + bg) * (x Wu^T + bu) of dense matrices
  backward   fh_gated_backward: the gradients of x, both weights and both biases
  step       layers.gated_linear forward and backward: the training step of such a layer

A stored matrix of R rows and C columns is one buffer: R rows of codes, a signed byte a value, padded with zeros to a
multiple of 128 columns, then R scales in binary32.
"""
from __future__ import annotations

import math

import torch

own = False

_DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
_SIZE = {"f32": 4, "bf16": 2}
_LEAST = 2.0 ** -100


# ---- the cases ---------------------------------------------------------------------------------------
def listed():
    return [
        # the smallest call: a handful of tokens' activations of an encoder (hidden 768), stored and restored
        {"name": "quantise_tokens", "kind": "quantise", "rows": 17, "cols": 768, "dtype": "bf16"},
        # a gated layer's output for a whole batch (16 x 512 tokens): the operand of the projection behind it
        {"name": "quantise_hidden", "kind": "quantise", "rows": 8192, "cols": 2048, "dtype": "bf16"},
        # one token through the projection back from a hidden width of 8192, weights stored once
        {"name": "product_token", "kind": "product", "m": 1, "n": 4096, "k": 8192, "out": "bf16", "bias": False},
        # a short prompt of ragged sizes
        {"name": "product_prompt", "kind": "product", "m": 197, "n": 1000, "k": 1537, "out": "f32", "bias": True},
        # the largest product: a wide layer over a long batch
        {"name": "product_large", "kind": "product", "m": 8192, "n": 8192, "k": 4096, "out": "bf16", "bias": True},
        # one token through a frozen gated layer, and a prompt of ragged sizes
        {"name": "serve_token", "kind": "serve", "tokens": 1, "features": 4096, "hidden": 8192, "act": "silu", "bias": False, "dtype": "bf16"},
        {"name": "serve_prompt", "kind": "serve", "tokens": 509, "features": 1023, "hidden": 2731, "act": "gelu", "bias": True, "dtype": "bf16"},
        # a few tokens through the layer as it is trained: an evaluation between steps
        {"name": "gated_tokens", "kind": "gated", "tokens": 4, "features": 4096, "hidden": 8192, "act": "silu", "bias": False, "dtype": "bf16"},
        # the forward pass of an encoder's feed-forward half (hidden 768) over a batch
        {"name": "gated_encoder", "kind": "gated", "tokens": 8192, "features": 768, "hidden": 2048, "act": "gelu", "bias": True, "dtype": "bf16"},
        # a small model's training step in fp32, every size odd
        {"name": "step_odd", "kind": "step", "tokens": 333, "features": 515, "hidden": 1001, "act": "gelu_tanh", "bias": True, "dtype": "f32"},
        # the encoder's training step
        {"name": "step_encoder", "kind": "step", "tokens": 8192, "features": 768, "hidden": 2048, "act": "gelu", "bias": True, "dtype": "bf16"},
        # the largest backward pass: a wide model's layer
        {"name": "backward_wide", "kind": "backward", "tokens": 4096, "features": 4096, "hidden": 8192, "act": "silu", "bias": False, "dtype": "bf16"},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(("quantise", "product", "product", "serve", "serve", "gated", "gated", "backward", "backward", "step"))
    case = {"kind": kind}
    if kind == "quantise":
        case["cols"] = _log(rng, 16, 16384)
        case["rows"] = min(_log(rng, 1, 16384), (1 << 24) // case["cols"])
        case["dtype"] = rng.choice(("f32", "bf16"))
    elif kind == "product":
        case.update(m=_log(rng, 1, 8192), n=_log(rng, 16, 8192), k=_log(rng, 16, 8192), out=rng.choice(("f32", "bf16")), bias=rng.random() < 0.5)
        case["k"] = min(case["k"], (1 << 38) // (case["m"] * case["n"]))
    else:
        # serving: from single tokens to a prompt; training in fp32 is for small models
        case["dtype"] = rng.choice(("f32", "bf16"))
        wide = kind == "serve" or case["dtype"] == "bf16"
        case.update(tokens=_log(rng, 1, 512 if kind == "serve" else 8192 if wide else 2048), features=_log(rng, 16, 4096 if wide else 1024),
                    hidden=_log(rng, 16, 8192 if wide else 2048), act=rng.choice(("silu", "gelu", "gelu_tanh")), bias=rng.random() < 0.5)
        case["tokens"] = min(case["tokens"], (1 << 37) // (case["features"] * case["hidden"]))
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


def _weights(g, n, k, dtype=torch.float32):
    return (torch.randn((n, k), generator=g, device="cuda") / math.sqrt(k)).to(dtype)


def _bias(g, n, wanted, dtype=torch.float32):
    return (0.2 * torch.randn(n, generator=g, device="cuda")).to(dtype) if wanted else None


def _padded(cols):
    return -(-cols // 128) * 128


def _stored(x):
    """The stored form of x, as a program holds a layer's weights or an operand that an earlier call left."""
    code, scale = _codes(x)
    return torch.cat((torch.nn.functional.pad(code, (0, _padded(x.shape[1]) - x.shape[1])).to(torch.int8).reshape(-1).view(torch.uint8),
                      scale.reshape(-1).view(torch.uint8)))


def prepare(case, seed):
    kind = case["kind"]
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    state = {"case": case}
    if kind == "quantise":
        state["x"] = _activation(g, case["rows"], case["cols"], _DTYPES[case["dtype"]])
        return state
    if kind == "product":
        state["a"] = _stored(_activation(g, case["m"], case["k"], torch.float32))
        state["b"] = _stored(_weights(g, case["n"], case["k"]))
        state["bias"] = _bias(g, case["n"], case["bias"])
        return state
    dtype, t, k, f = _DTYPES[case["dtype"]], case["tokens"], case["features"], case["hidden"]
    state["x"] = _activation(g, t, k, dtype)
    if kind == "serve":
        state["wg"], state["wu"] = _stored(_weights(g, f, k)), _stored(_weights(g, f, k))
    else:
        state["wg"], state["wu"] = _weights(g, f, k, dtype), _weights(g, f, k, dtype)
    state["bg"], state["bu"] = _bias(g, f, case["bias"], dtype), _bias(g, f, case["bias"], dtype)
    if kind in ("backward", "step"):
        state["dh"] = _gradient(g, t, f, dtype)
    if kind == "step":
        for name in ("x", "wg", "wu", "bg", "bu"):
            if state[name] is not None:
                state[name].requires_grad_()
    return state


# ---- the plain forms: torch operations in 32 bits --------------------------------------------------------
def _codes(x):
    """(whole numbers -127 .. 127, the scale of every row)"""
    x = x.float()
    top = x.abs().amax(1, keepdim=True)
    some = top >= _LEAST
    times = torch.where(some, 127.0 / top, 0.0)
    return torch.round(x * times), torch.where(some, top / 127.0, 0.0)


def _values(buffer, rows, cols):
    """The values that a stored matrix stands for, in 32 bits."""
    width = _padded(cols)
    codes = buffer[:rows * width].view(torch.int8).view(rows, width)[:, :cols]
    return codes.float() * buffer[rows * width:].view(torch.float32)[:, None]


def _activated(g, act):
    """(act(g), its derivative)"""
    if act == "silu":
        s = torch.sigmoid(g)
        return g * s, s * (1.0 + g * (1.0 - s))
    if act == "gelu":
        part = 0.5 * (1.0 + torch.erf(g * math.sqrt(0.5)))
        return g * part, part + g * torch.exp(-0.5 * g * g) / math.sqrt(2.0 * math.pi)
    c = math.sqrt(2.0 / math.pi)
    t = torch.tanh(c * (g + 0.044715 * g * g * g))
    return 0.5 * g * (1.0 + t), 0.5 * (1.0 + t) + 0.5 * g * (1.0 - t * t) * c * (1.0 + 3.0 * 0.044715 * g * g)


def _linear(x, w, bias):
    y = x @ w.t()
    return y if bias is None else y + bias.float()


def _rounded(values, dtype):
    return [None if v is None else v.to(dtype) for v in values]


def _run_plain(state):
    case, kind = state["case"], state["case"]["kind"]
    if kind == "quantise":
        code, scale = _codes(state["x"])
        return (code * scale).to(state["x"].dtype)
    if kind == "product":
        return _linear(_values(state["a"], case["m"], case["k"]), _values(state["b"], case["n"], case["k"]), state["bias"]).to(_DTYPES[case["out"]])
    dtype, act = _DTYPES[case["dtype"]], case["act"]
    if kind == "serve":
        code, scale = _codes(state["x"])
        x = code * scale
        wg, wu = (_values(state[w], case["hidden"], case["features"]) for w in ("wg", "wu"))
        return (_activated(_linear(x, wg, state["bg"]), act)[0] * _linear(x, wu, state["bu"])).to(dtype)
    with torch.no_grad():
        x, wg, wu = state["x"].float(), state["wg"].float(), state["wu"].float()
        u = _linear(x, wu, state["bu"])
        a, slope = _activated(_linear(x, wg, state["bg"]), act)
        if kind == "gated":
            return (a * u).to(dtype)
        dh = state["dh"].float()
        dg, du = dh * u * slope, dh * a
        grads = [dg @ wg + du @ wu, dg.t() @ x, du.t() @ x]
        if case["bias"]:
            grads += [dg.sum(0), du.sum(0)]
        return _rounded(([a * u] if kind == "step" else []) + grads, dtype)


# ---- the framework's calls -------------------------------------------------------------------------------
def _run_own(state):
    from paper_2510_11400_amd import api, layers
    case, kind = state["case"], state["case"]["kind"]
    if kind == "quantise":
        return api.fh_q8_dequantize(api.fh_q8_quantize(state["x"]), out_dtype=state["x"].dtype)
    if kind == "product":
        a = api.Q8Matrix(state["a"], case["m"], case["k"])
        b = api.Q8Matrix(state["b"], case["n"], case["k"])
        return api.fh_q8_matmul(a, b, bias=state["bias"], out_dtype=_DTYPES[case["out"]])
    biases = {"b_gate": state["bg"], "b_up": state["bu"]}
    if kind == "serve":
        wg, wu = (api.Q8Matrix(state[w], case["hidden"], case["features"]) for w in ("wg", "wu"))
        return api.fh_q8_gated(api.fh_q8_quantize(state["x"]), wg, wu, activation=case["act"], out_dtype=state["x"].dtype, **biases)
    weights = (state["x"], state["wg"], state["wu"])
    if kind == "gated":
        return api.fh_gated(*weights, activation=case["act"], **biases)
    if kind == "backward":
        grads = api.fh_gated_backward(state["dh"], *weights, activation=case["act"], **biases)
        return list(grads if case["bias"] else grads[:3])
    leaves = [*weights, *((state["bg"], state["bu"]) if case["bias"] else ())]
    h = layers.gated_linear(*weights, activation=case["act"], **biases)
    return [h.detach(), *torch.autograd.grad(h, leaves, state["dh"])]


def run(state):
    return _run_own(state) if own else _run_plain(state)


# ---- what a pass cannot do without ---------------------------------------------------------------------
def _stored_bytes(rows, cols):
    return rows * cols + 4 * rows


def work(case):
    """Every input read once, every output written once; what is stored in between is written and read back."""
    kind = case["kind"]
    if kind == "quantise":
        n = case["rows"] * case["cols"]
        return {"bytes": 2 * n * _SIZE[case["dtype"]] + 2 * _stored_bytes(case["rows"], case["cols"]), "flops": 4 * n}
    if kind == "product":
        m, n, k = case["m"], case["n"], case["k"]
        return {"bytes": _stored_bytes(m, k) + _stored_bytes(n, k) + m * n * _SIZE[case["out"]], "flops": 2 * m * n * k}
    t, k, f, size = case["tokens"], case["features"], case["hidden"], _SIZE[case["dtype"]]
    if kind == "serve":
        return {"bytes": size * (t * k + t * f) + 2 * _stored_bytes(t, k) + 2 * _stored_bytes(f, k), "flops": 4 * t * k * f}
    forward = {"bytes": size * (t * k + 2 * f * k + t * f), "flops": 4 * t * k * f}
    if kind == "gated":
        return forward
    # backward: x, dh and both weights in, their gradients out; g and u are computed again where the call is given no more than that
    backward = {"bytes": size * (2 * t * k + 4 * f * k + t * f), "flops": 12 * t * k * f}
    if kind == "backward":
        return backward
    return {"bytes": forward["bytes"] + backward["bytes"], "flops": 12 * t * k * f}


# ---- the same in binary64 ------------------------------------------------------------------------------
def _f32(x):
    """Binary64 rounded to the nearest binary32, as binary64."""
    return x.to(torch.float32).double()


def _codes64(x):
    """The stored form's definition: its scale, factor and product are binary32 numbers by definition."""
    code, scale = torch.zeros_like(x), torch.zeros((x.shape[0], 1), dtype=torch.float64, device=x.device)
    top = x.abs().max(1).values
    for rows in torch.nonzero(top >= _LEAST).view(-1).split(4096):
        code[rows] = torch.special.round(_f32(x[rows] * _f32(127.0 / top[rows])[:, None]))
        scale[rows, 0] = _f32(top[rows] / 127.0)
    return code, scale


def _decoded64(buffer, rows, cols):
    width = _padded(cols)
    n = buffer[:rows * width].view(rows, width)[:, :cols].double()
    n = torch.where(n >= 128, n - 256, n)                        # a signed byte
    return n, buffer[rows * width:].view(torch.float32).double()


def _activated64(g, act):
    if act == "silu":
        return g / (1.0 + torch.exp(-g))
    if act == "gelu":
        return g * torch.special.erfc(-g / math.sqrt(2.0)) / 2.0
    return g * torch.special.expit(math.sqrt(8.0 / math.pi) * (g + 0.044715 * g ** 3))


def exact(case, seed):
    kind, state = case["kind"], prepare(case, seed)
    if kind == "quantise":
        code, scale = _codes64(state["x"].double())
        return code * scale
    if kind == "product":
        a, sa = _decoded64(state["a"], case["m"], case["k"])
        b, sb = _decoded64(state["b"], case["n"], case["k"])
        y = torch.mm(a, b.t()) * (sa[:, None] * sb[None, :])
        return y if state["bias"] is None else y + state["bias"].double()
    biases = [None if state[b] is None else state[b].detach().double() for b in ("bg", "bu")]
    if kind == "serve":
        code, scale = _codes64(state["x"].double())
        parts = []
        for name, bias in zip(("wg", "wu"), biases):
            w, sw = _decoded64(state[name], case["hidden"], case["features"])
            y = torch.mm(code, w.t()) * (scale * sw[None, :])
            parts.append(y if bias is None else y + bias)
        return _activated64(parts[0], case["act"]) * parts[1]
    leaves = [state[name].detach().double() for name in ("x", "wg", "wu")] + [b for b in biases if b is not None]
    for leaf in leaves:
        leaf.requires_grad_(kind != "gated")
    x, wg, wu = leaves[:3]
    g, u = torch.mm(x, wg.t()), torch.mm(x, wu.t())
    if case["bias"]:
        g, u = g + leaves[3], u + leaves[4]
    h = _activated64(g, case["act"]) * u
    if kind == "gated":
        return h
    grads = torch.autograd.grad(h, leaves, state["dh"].double())
    return [h.detach(), *grads] if kind == "step" else list(grads)
